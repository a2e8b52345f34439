// ccq_policy.cu -- clipped policy loss with a KL term over token logits, its gradient, and the token
// log-probabilities alone (ccq_ops.h).
//
// For a row x of logits with maximum m, e_j = exp((x_j - m) / T), Z = sum e_j, the row's log-probability is
//   logp = (x_a - m) / T - log Z
// and everything else is a function of the row's scalars; the gradient is
//   dlogits_j = c (delta_ja - e_j / Z),   c = grad_scale w dL/dlogp / T,
//   dL/dlogp = -(r A where r A <= clip(r) A, else 0) + kl_coef (1 - exp(ref - logp)).
// policy_staged_kernel reads each logit once: a row stays in the shared memory of a cluster, its exponentials in
// registers, until its sum is known, and the gradient leaves by the way the logits came.  Rows beyond what 16 CTAs
// hold (vocabularies above 520 thousand in bf16, 260 thousand in fp32) go through policy_row_kernel, which reads them
// twice.  policy_loss_kernel adds the rows' losses.
// HBM bounds it: 8192 x 32000 bf16, a quarter masked (918 MB): 154 us, 6.0 TB/s, 88 % of the copy rate; 1500 x 128001 (rows on
// no 16-byte boundary, 742 MB): 135 to 137 us, 80 %.  Short rows are bound by a row's chain of reductions (8192 x 3500: 58 %),
// rows over several CTAs also by how many clusters fit the groups of SMs (512 x 200000 fp32: 67 %).
#include <algorithm>

#include "ccq_ops.cuh"

namespace ccq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct PolicyArgs {
    const void *logits, *actions;
    int64_t logits_stride, dlogits_stride, n;
    int id_bytes, vocab;
    const float *old_logp, *ref_logp, *advantages, *weights;
    ccq_policy_params p;
    float scale;        // log2(e) / temperature
    float inv, inv_lo;  // 1 / temperature, as a sum
    float grad_mul;     // grad_scale / temperature
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

struct RowScalars {
    int action;
    int row;  // of a batch
    float weight, adv, old, ref, chosen;  // chosen: the action's logit
};

// Whether the row is not masked; its weight and action are read together.
__device__ __forceinline__ bool is_live(const PolicyArgs &a, int64_t i) {
    const float w = a.weights ? a.weights[i] : 1.f;
    const int64_t t = load_index(a.actions, a.id_bytes, i);
    return w != 0.f && t >= 0 && t < a.vocab;
}

// The log-probability (chosen - m) / T - log z as the sum of two floats.  The loss needs its differences from the old and
// reference ones to more than its own rounding: at logp = -8 that is 5e-7, which a KL term with d = 1e-3 sees 1000-fold.
// (Knuth's exact difference; log z = e log 2 + log f with the high part of log 2 short enough for an exact product, after
// Cody and Waite.  Each of these roundings is an operation of its own: a product fused into the sum behind it would leave
// in the low part what r has already.)
struct TwoFloats {
    float hi, lo;
};
__device__ __forceinline__ TwoFloats exact_sum(float a, float b) {
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ TwoFloats log_probability(float chosen, float m, float z, float inv, float inv_lo) {
    const TwoFloats diff = exact_sum(chosen, -m);
    const float q = __fmul_rn(diff.hi, inv);
    // no digits below an infinity (a masked action, also one at the type's lowest value once the temperature has divided it)
    if (!(fabsf(q) < INFINITY)) return {q - logf(z), 0.f};
    const float r = fmaf(diff.hi, inv_lo, fmaf(diff.lo, inv, fmaf(diff.hi, inv, -q)));
    const int e = (static_cast<int>(__float_as_uint(z)) - 0x3f400000) >> 23;  // z = 2^e f, f in [0.75, 1.5)
    const float f = __uint_as_float(__float_as_uint(z) - (static_cast<uint32_t>(e) << 23)), k = static_cast<float>(e);
    const TwoFloats s = exact_sum(q, __fmul_rn(-k, 0.693115234375f));
    const float rest = (r + s.lo) - fmaf(k, 3.19461849453e-05f, logf(f) + (z - z));  // (z - z: not a number stays one)
    return exact_sum(s.hi, rest);
}

// The row's loss and c of the gradient, from its log-probability.
__device__ __forceinline__ float row_loss(const PolicyArgs &a, const RowScalars &r, TwoFloats logp, float &c) {
    const float adv = r.adv;
    const float ratio = expf((logp.hi - r.old) + logp.lo);
    const float open = ratio * adv;
    const float held = fminf(fmaxf(ratio, 1.f - a.p.clip_low), 1.f + a.p.clip_high) * adv;
    // a ratio or advantage that is not a number stays one
    float loss = open <= held || !(held < open) ? -open : -held;
    float slope = open <= held || !(held < open) ? -open : 0.f;
    if (a.ref_logp && a.p.kl_coef != 0.f) {
        const float d = (r.ref - logp.hi) - logp.lo;
        const float em1 = expm1f(d);
        loss += a.p.kl_coef * (em1 < INFINITY ? em1 - d : em1);  // (infinite d: exp(d) outgrows it)
        slope -= a.p.kl_coef * em1;
    }
    c = r.weight * slope * a.grad_mul;
    return r.weight * loss;
}

constexpr int kRowThreads = 512;

// Two (maximum, sum) pairs to one.
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
            const TwoFloats logp = log_probability(to_f32(x[row.action]), m, z, a.inv, a.inv_lo);
            float c = 0.f;
            if (a.score) {
                a.logp[i] = logp.hi;
            } else {
                RowScalars r = {};
                r.weight = row.weight;
                r.adv = a.advantages[i];
                r.old = a.old_logp[i];
                if (a.ref_logp) r.ref = a.ref_logp[i];
                a.row_loss[i] = row_loss(a, r, logp, c);
                if (a.logp) a.logp[i] = logp.hi;
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

// ---------------------------------------------------------------- rows in shared memory

// A cluster of `cs` CTAs takes a row, each a slice of its 16-byte granules, in one of three to kMaxBuffers buffers of
// shared memory: while a row is computed, the next ones come in and the gradients of the ones before, written over
// their logits, go out, both as bulk copies.  Each logit is read from memory once.  A row that starts or ends inside a
// granule (an odd vocabulary) has those elements fetched one by one a row ahead, and what belongs to its neighbours
// replaced by -inf; the gradient's first and last elements are stored one by one.
constexpr int kMaxBuffers = 8;  // (8192 x 3500 bf16: 3 to 8 of them 31 to 33 us, 8192 x 8000 53 to 56: little, and more cost nothing)
// Rows whose scalars a CTA holds at once: the more CTAs share an SM, the fewer.
constexpr int batch_rows(int threads) { return threads <= 128 ? 64 : 256; }
constexpr int kMaxCluster = 16;
constexpr int kRanked = 16384;
constexpr int kGranules = 8;  // of a thread: their exponentials stay in registers until the row's sum is known
constexpr size_t kSmBytes = 206848;  // shared memory that the CTAs of an SM divide among them
constexpr float kLowest = -3.402823466e38f;

struct Staging {
    int per;  // granules of a slice
    int cs, buffers;
    int ranked;  // rows are dealt out by their rank among the live ones
    int64_t clusters;
    int64_t span;  // rows dealt out at a time, at most batch_rows() to a cluster
};

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// Writes v to p in CTA `cta` of the cluster and tells that CTA's barrier of the 8 bytes.
__device__ __forceinline__ void tell_peer(float2 *p, uint64_t *bar, int cta, float2 v) {
    uint32_t to, at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(p)), "r"(cta));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(bar)), "r"(cta));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(to),
                 "l"(f2_make(v.x, v.y)), "r"(at)
                 : "memory");
}

// mbar_wait for a barrier that the cluster's other CTAs complete.
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t *bar, uint32_t parity, volatile int *abort, int *status) {
    const long long start = clock64();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_addr(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if (*abort) return false;
        if (clock64() - start > kWaitLimitCycles) {
            *abort = 1;
            atomicExch(status, kStatusTimeout);
            return false;
        }
    }
}

// (maximum, sum) pairs of a warp's lanes to those of all of them.  A sum is scaled to the common maximum; equal maxima
// keep theirs as it is.
__device__ __forceinline__ void join_warp(float &m, float &z, float scale) {
    float top = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    z *= fast_exp2((m - top) * scale);
#pragma unroll
    for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(~0u, z, o);
    m = top;
}

// The larger of each pair of packed bf16 values (numbers before NaN; a NaN shows in the sum).
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// The largest of a thread's granules.
template <typename T> __device__ __forceinline__ float granules_max(const uint4 (&r)[kGranules]) {
    if constexpr (IsBf16<T>::value) {
        uint32_t m = r[0].x;
#pragma unroll
        for (int q = 0; q < kGranules; ++q) m = max_bf16x2(m, max_bf16x2(max_bf16x2(r[q].x, r[q].y), max_bf16x2(r[q].z, r[q].w)));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    } else {
        float m = kLowest;
#pragma unroll
        for (int q = 0; q < kGranules; ++q)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(r[q].x), __uint_as_float(r[q].y)),
                               fmaxf(__uint_as_float(r[q].z), __uint_as_float(r[q].w))));
        return m;
    }
}

// A granule's values as pairs, exp2((x - m) scale).
template <typename T> __device__ __forceinline__ void granule_exp(const uint4 &r, uint64_t minus_m, uint64_t scale, uint64_t *e) {
    constexpr int kPairs = IsBf16<T>::value ? 4 : 2;
    uint64_t x[kPairs];
    if constexpr (IsBf16<T>::value) {
        x[0] = f2_from_bf16x2(r.x);
        x[1] = f2_from_bf16x2(r.y);
        x[2] = f2_from_bf16x2(r.z);
        x[3] = f2_from_bf16x2(r.w);
    } else {
        x[0] = f2_make(__uint_as_float(r.x), __uint_as_float(r.y));
        x[1] = f2_make(__uint_as_float(r.z), __uint_as_float(r.w));
    }
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const float2 d = f2_split(f2_mul(f2_add(x[i], minus_m), scale));
        e[i] = f2_make(fast_exp2(d.x), fast_exp2(d.y));
    }
}

template <typename T, int THREADS, int GRAD>
__global__ void __launch_bounds__(THREADS, 512 / THREADS) policy_staged_kernel(PolicyArgs a, Staging g) {
    constexpr int N = 16 / static_cast<int>(sizeof(T));
    constexpr int kPairs = N / 2;
    constexpr int kWarps = THREADS / 32, kBatch = batch_rows(THREADS);
    extern __shared__ __align__(128) uint8_t dyn[];  // [buffers][per] granules, then the batch's scalars
    __shared__ uint64_t full[kMaxBuffers], heard[2];
    __shared__ int give_up;
    __shared__ float2 pairs[kWarps];
    __shared__ __align__(8) float2 peers[2][kMaxCluster];
    __shared__ uint32_t live_bits[kBatch / 32], dead_bits[kBatch / 32];
    __shared__ int live_rows[kBatch], dead_rows[kBatch], counts[2], warp_live[kWarps];
    __shared__ uint32_t row_bits[THREADS == 512 ? kRanked / 32 : 1];
    RowScalars *list = reinterpret_cast<RowScalars *>(dyn + static_cast<size_t>(g.buffers) * g.per * 16);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = static_cast<int>(blockIdx.x % g.cs);
    const int64_t cluster = blockIdx.x / g.cs;
    if (tid == 0) {
        for (int b = 0; b < kMaxBuffers; ++b) mbar_init(&full[b], 1);
        for (int b = 0; b < 2; ++b) mbar_init(&heard[b], 1);
        give_up = 0;
        fence_barrier_init();
    }
    __syncthreads();
    if (g.cs > 1) cluster_barrier();  // every CTA of the cluster runs before its shared memory is written
    const T *logits = static_cast<const T *>(a.logits);
    T *dlogits = static_cast<T *>(a.dlogits);
    const int first = rank * g.per;  // this slice's first granule
    // rows loaded (thread 0) and computed so far: their buffers and the barriers' phases
    uint32_t load_at = 0, at = 0, phase = 0, rows = 0, issued = 0;
    // rows whose gradients may still be leaving (with more than three buffers 1 or 2: 8192 x 3500 32.4 and 31.4 us, 8192 x 8000
    // the same; with three, 2 leaves one row's loads ahead: 8192 x 32000 159 and 247 us)
    const int lag = g.buffers > 3 ? 2 : 1;
    const int ahead = g.buffers - lag;      // rows whose logits are under way or here

    // Elements of row i before its first granule's start, and the granules it touches.
    auto offset_of = [](const void *row) { return static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)); };
    auto buffer = [&](uint32_t b) { return reinterpret_cast<uint4 *>(dyn) + static_cast<size_t>(b) * g.per; };
    auto slice_end = [&](int granules) { return granules - first < g.per ? granules - first : g.per; };
    // Thread 0: the whole granules of row i's slice into the next buffer.
    auto load_row = [&](int64_t i) {
        const T *row = logits + i * a.logits_stride;
        const int off = offset_of(row), whole = (off + a.vocab) / N;
        const int lo = first > 0 || off == 0 ? 0 : 1, hi = slice_end(whole);
        const uint32_t b = load_at;
        if (hi > lo) {
            mbar_arrive_expect_tx(&full[b], static_cast<uint32_t>(hi - lo) * 16);
            bulk_load(buffer(b) + lo, row - off + static_cast<int64_t>(first + lo) * N, static_cast<uint32_t>(hi - lo) * 16, &full[b]);
        } else {
            mbar_arrive(&full[b]);
        }
        load_at = load_at + 1 == static_cast<uint32_t>(g.buffers) ? 0 : load_at + 1;
        ++issued;
    };
    // The last warp's lanes: the elements of the granules that row i shares with its neighbours, -inf in the others' places.
    // `cell` is where the value belongs in the row's buffer (-1: nowhere in this slice).
    auto edge_of = [&](int64_t i, int &cell) {
        const T *row = logits + i * a.logits_stride;
        const int off = offset_of(row), granules = (off + a.vocab + N - 1) / N;
        const int tail = (off + a.vocab) % N;
        cell = -1;
        T v = from_f32<T>(-INFINITY);
        const int e = lane % N, side = lane / N;
        if (warp != kWarps - 1 || side > 1) return v;
        int at = -1;  // granule
        if (side == 0 && off) at = 0;
        if (side == 1 && tail && !(granules == 1 && off)) at = granules - 1;
        if (at < first || at >= first + slice_end(granules)) return v;
        cell = (at - first) * N + e;
        const int64_t c = static_cast<int64_t>(at) * N + e - off;
        if (c >= 0 && c < a.vocab) v = row[c];
        return v;
    };

    // A later bulk copy writes over these cells when the buffer comes round, so the ordinary store is ordered before the copies
    // that the next barrier lets thread 0 start.  (With a gradient the fence that every thread makes in the row itself does that.)
    auto set_edge = [&](uint4 *buf, int cell, T v) {
        if (cell < 0) return;
        reinterpret_cast<T *>(buf)[cell] = v;
        if constexpr (!GRAD) fence_proxy_async_smem();
    };

    for (int64_t start = 0; start < a.n; start += g.span) {
        // this cluster's rows of the span: `live` ones to compute and `dead` (masked) ones to zero
        const int64_t span = a.n - start < g.span ? a.n - start : g.span;
        if (tid < 2) counts[tid] = 0;
        __syncthreads();
        if (THREADS == 512 && g.ranked) {
            // a bit for each row of the span, the live rows before each word of them, then every cluster takes each
            // clusters-th of the live rows, and of the dead
            const int words = static_cast<int>((span + 31) / 32);
            for (int w = warp; w < words; w += kWarps * 4) {
                bool live[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t k = static_cast<int64_t>(w + q * kWarps) * 32 + lane;
                    live[q] = k < span && is_live(a, start + k);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t bits = __ballot_sync(~0u, live[q]);
                    if (lane == 0 && w + q * kWarps < words) row_bits[w + q * kWarps] = bits;
                }
            }
            __syncthreads();
            constexpr int kEach = (kRanked / 32 + THREADS - 1) / THREADS;  // words of a thread
            int alive = 0;
#pragma unroll
            for (int q = 0; q < kEach; ++q)
                if (tid * kEach + q < words) alive += __popc(row_bits[tid * kEach + q]);
            int before = alive;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int t = __shfl_up_sync(~0u, before, o);
                if (lane >= o) before += t;
            }
            if (lane == 31) warp_live[warp] = before;
            __syncthreads();
            before -= alive;
            int all = 0;
            for (int w = 0; w < kWarps; ++w) {
                if (w < warp) before += warp_live[w];
                all += warp_live[w];
            }
            const int c = static_cast<int>(cluster), cs = static_cast<int>(g.clusters);
            for (int q = 0; q < kEach; ++q) {
                const int w = tid * kEach + q;
                if (w >= words) break;
                const uint32_t bits = row_bits[w];
                const int here = span - w * 32 < 32 ? static_cast<int>(span) - w * 32 : 32;
                // the first live row at or after `before`, and the first dead one, that are this cluster's
                for (int r = before + (c - before % cs + cs) % cs; r < before + __popc(bits); r += cs)
                    live_rows[r / cs] = w * 32 + __fns(bits, 0, r - before + 1);
                const int gone = w * 32 - before;
                const uint32_t none = ~bits & (here < 32 ? (1u << here) - 1 : ~0u);
                for (int r = gone + (c - gone % cs + cs) % cs; r < gone + __popc(none); r += cs)
                    dead_rows[r / cs] = w * 32 + __fns(none, 0, r - gone + 1);
                before += __popc(bits);
            }
            if (tid == 0) {
                counts[0] = all > c ? (all - c + cs - 1) / cs : 0;
                counts[1] = static_cast<int>(span) - all > c ? (static_cast<int>(span) - all - c + cs - 1) / cs : 0;
            }
        } else {
            // every clusters-th row
            for (int q = 0; q < kBatch; q += THREADS) {
                const int k = q + tid;
                const int64_t at = cluster + k * g.clusters;
                const bool here = k < kBatch && at < span, live = here && is_live(a, start + at);
                const uint32_t l = __ballot_sync(~0u, live), d = __ballot_sync(~0u, here && !live);
                if (lane == 0 && k < kBatch) {
                    live_bits[k >> 5] = l;
                    dead_bits[k >> 5] = d;
                }
            }
            __syncthreads();
            for (int k = tid; k < kBatch; k += THREADS) {
                const int w = k >> 5, bit = k & 31;
                const bool live = (live_bits[w] >> bit) & 1;
                if (!live && !((dead_bits[w] >> bit) & 1)) continue;
                const uint32_t *bits = live ? live_bits : dead_bits;
                int at = __popc(bits[w] & ((1u << bit) - 1));
                for (int v = 0; v < w; ++v) at += __popc(bits[v]);
                (live ? live_rows : dead_rows)[at] = static_cast<int>(cluster + k * g.clusters);
            }
            if (tid < 2) {
                int all = 0;
                for (int v = 0; v < kBatch / 32; ++v) all += __popc(tid ? dead_bits[v] : live_bits[v]);
                counts[tid] = all;
            }
        }
        __syncthreads();
        const int count = counts[0], dead = counts[1];
        for (int k = tid; k < count; k += THREADS) {
            const int64_t i = start + live_rows[k];
            const Row r = row_of(a, i, false);
            RowScalars sc;
            sc.action = r.action;
            sc.row = live_rows[k];
            sc.weight = r.weight;
            sc.chosen = to_f32(logits[i * a.logits_stride + r.action]);
            sc.adv = a.score ? 0.f : a.advantages[i];
            sc.old = a.score ? 0.f : a.old_logp[i];
            sc.ref = a.ref_logp ? a.ref_logp[i] : 0.f;
            list[k] = sc;
        }
        for (int k = tid; k < dead && rank == 0; k += THREADS) {
            const int64_t i = start + dead_rows[k];
            row_of(a, i, true);
            if (a.logp) a.logp[i] = a.score ? __int_as_float(0x7fc00000) : 0.f;
            if (!a.score) a.row_loss[i] = 0.f;
        }
        __syncthreads();
        auto row_index = [&](int j) { return start + list[j].row; };
        if (tid == 0)
            for (int j = 0; j < ahead && j < count; ++j) load_row(row_index(j));
        if (count > 0) {
            int cell;
            const T v = edge_of(row_index(0), cell);
            set_edge(buffer(at), cell, v);
        }
        if constexpr (GRAD) {
            // masked rows: zeros, while the first rows come in
            for (int k = 0; k < dead; ++k) {
                T *row = dlogits + (start + dead_rows[k]) * a.dlogits_stride;
                const int off = offset_of(row), granules = (off + a.vocab + N - 1) / N;
                for (int c = tid; c < slice_end(granules); c += THREADS) {
                    const int64_t e = static_cast<int64_t>(first + c) * N - off;
                    if (e >= 0 && e + N <= a.vocab) {
                        __stcs(reinterpret_cast<uint4 *>(row + e), make_uint4(0, 0, 0, 0));
                    } else {
                        for (int q = 0; q < N; ++q)
                            if (e + q >= 0 && e + q < a.vocab) row[e + q] = from_f32<T>(0.f);
                    }
                }
            }
        }
        __syncthreads();
        for (int j = 0; j < count; ++j, ++rows) {
            const RowScalars sc = list[j];
            const int64_t i = start + sc.row;
            const T *row = logits + i * a.logits_stride;
            const int off = offset_of(row), granules = (off + a.vocab + N - 1) / N, mygran = slice_end(granules);
            const uint32_t next = at + 1 == static_cast<uint32_t>(g.buffers) ? 0 : at + 1;
            uint4 *buf = buffer(at);
            int edge_cell = -1;
            T edge = from_f32<T>(0.f);
            if (j + 1 < count) edge = edge_of(row_index(j + 1), edge_cell);
            if (g.cs > 1 && tid == 0) mbar_arrive_expect_tx(&heard[rows & 1], static_cast<uint32_t>(g.cs) * 8);
            mbar_wait(&full[at], phase, &give_up, a.status);
            // this thread's exponentials, against its own maximum, and their sum
            constexpr uint32_t low = IsBf16<T>::value ? 0xff80ff80u : 0xff800000u;  // -inf
            const uint64_t scale = f2_make(a.scale, a.scale);
            uint64_t e[kGranules][kPairs];
            float m, z;
            {
                uint4 r[kGranules];
#pragma unroll
                for (int q = 0; q < kGranules; ++q) {
                    r[q] = make_uint4(low, low, low, low);
                    if (q * THREADS + tid < mygran) r[q] = buf[q * THREADS + tid];
                }
                m = fmaxf(granules_max<T>(r), kLowest);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int q = 0; q < kGranules; ++q) {
                    granule_exp<T>(r[q], f2_make(-m, -m), scale, e[q]);
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) sum[k & 1] = f2_add(sum[k & 1], e[q][k]);
                }
                const float2 t = f2_split(f2_add(sum[0], sum[1]));
                z = t.x + t.y;
            }
            const float own = m;
            join_warp(m, z, a.scale);
            if (lane == 0) pairs[warp] = make_float2(m, z);
            __syncthreads();
            const bool alone = g.cs == 1;
            if (alone || warp == 0) {
                const float2 p = lane < kWarps ? pairs[lane] : make_float2(kLowest, 0.f);
                m = p.x;
                z = p.y;
                join_warp(m, z, a.scale);
            }
            if (!alone) {
                // (a CTA tells its row after the next only when all have told the next, so two sets of cells do)
                if (warp == 0 && lane < g.cs) tell_peer(&peers[rows & 1][rank], &heard[rows & 1], lane, make_float2(m, z));
                mbar_wait_cluster(&heard[rows & 1], (rows >> 1) & 1, &give_up, a.status);
                const float2 p = lane < g.cs ? peers[rows & 1][lane] : make_float2(kLowest, 0.f);
                m = p.x;
                z = p.y;
                join_warp(m, z, a.scale);
            }
            const TwoFloats logp = log_probability(sc.chosen, m, z, a.inv, a.inv_lo);
            float c1 = 0.f, loss = 0.f;
            if (!a.score) loss = row_loss(a, sc, logp, c1);
            if (rank == 0 && tid == 0) {
                if (a.logp) a.logp[i] = logp.hi;
                if (!a.score) a.row_loss[i] = loss;
            }
            if constexpr (GRAD) {
                T *drow = dlogits + i * a.dlogits_stride;
                const bool direct = offset_of(drow) != off;  // the two rows lie differently over their granules
                const float c2 = -c1 / z, mine2 = c2 * fast_exp2((own - m) * a.scale);
                const uint64_t mul = f2_make(mine2, mine2);
                // local granules that are stored element by element: those shared with the neighbours, or all
                const int head = first == 0 && off ? 0 : -1, tail = (off + a.vocab) % N ? granules - 1 - first : -1;
#pragma unroll
                for (int q = 0; q < kGranules; ++q) {
                    const int c = q * THREADS + tid;
                    if (c >= mygran) continue;
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) e[q][k] = f2_mul(e[q][k], mul);
                    if (c != head && c != tail && !direct) {
                        uint4 o;
                        if constexpr (IsBf16<T>::value) {
                            o = make_uint4(bf16x2_from_f2(e[q][0]), bf16x2_from_f2(e[q][1]), bf16x2_from_f2(e[q][2]), bf16x2_from_f2(e[q][3]));
                        } else {
                            const float2 x = f2_split(e[q][0]), y = f2_split(e[q][1]);
                            o = make_uint4(__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(y.x), __float_as_uint(y.y));
                        }
                        buf[c] = o;
                    } else {
                        const int64_t el = static_cast<int64_t>(first + c) * N - off;
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            const float2 t = f2_split(e[q][k / 2]);
                            if (el + k >= 0 && el + k < a.vocab) drow[el + k] = from_f32<T>(k % 2 ? t.y : t.x);
                        }
                    }
                }
                // the action's element, by the thread that has just stored its granule
                const int at = sc.action + off - first * N, c = at / N;
                if (at >= 0 && c < mygran && c % THREADS == tid) {
                    const T v = from_f32<T>(c1 + c2 * fast_exp2((sc.chosen - m) * a.scale));
                    if (c != head && c != tail && !direct) reinterpret_cast<T *>(buf)[at] = v;
                    else drow[sc.action] = v;
                }
                fence_proxy_async_smem();
            }
            set_edge(buffer(next), edge_cell, edge);
            __syncthreads();
            if (tid == 0) {
                if constexpr (GRAD) {
                    T *drow = dlogits + i * a.dlogits_stride;
                    if (offset_of(drow) == off) {
                        const int whole = (off + a.vocab) / N, lo = first > 0 || off == 0 ? 0 : 1, hi = slice_end(whole);
                        if (hi > lo) bulk_store(drow - off + static_cast<int64_t>(first + lo) * N, buf + lo, static_cast<uint32_t>(hi - lo) * 16);
                    }
                    tma_store_commit();
                    // the row `lag` before this one has left the buffer that the next load takes
                    if (lag == 1) tma_store_wait_read_but<1>();
                    else tma_store_wait_read_but<2>();
                }
                if (j + ahead < count) load_row(row_index(j + ahead));
            }
            at = next;
            if (!at) phase ^= 1;
        }
        __syncthreads();  // the batch's scalars may go
    }
    if (tid == 0) {
        if constexpr (GRAD) tma_store_wait_all();
        // copies that a wait gave up on have landed too before the CTA leaves (all others have: no time)
        const uint32_t buffers = static_cast<uint32_t>(g.buffers);
        for (uint32_t b = 0; b < buffers; ++b)
            if (const uint32_t uses = (issued + buffers - 1 - b) / buffers) mbar_drain(&full[b], (uses - 1) & 1);
        if (g.cs > 1 && rows) mbar_drain(&heard[(rows - 1) & 1], ((rows - 1) >> 1) & 1);
    }
    if (g.cs > 1) cluster_barrier();  // no CTA leaves while others may still write to it
}

struct StagePlan {
    int threads, cs, per, buffers, clusters;  // clusters: those the device holds at once
    size_t smem;
};

int64_t row_granules(const PolicyArgs &a, int es) {
    const int n = 16 / es;
    return (static_cast<int64_t>(a.vocab) + 2 * (n - 1)) / n + 1;
}

// A plan for slices of a cs-th of a row: the fewest threads that hold one, and shared memory for as many buffers as
// an SM's 512 threads leave room for (short rows need more of them under way).
StagePlan slice_plan(int64_t granules, int cs) {
    StagePlan p = {};
    p.cs = cs;
    p.per = static_cast<int>((granules + cs - 1) / cs);
    p.threads = p.per <= 32 * kGranules ? 32 : p.per <= 64 * kGranules ? 64 : p.per <= 128 * kGranules ? 128 : p.per <= 256 * kGranules ? 256 : 512;
    const size_t scalars = batch_rows(p.threads) * sizeof(RowScalars);
    const size_t share = kSmBytes / (512 / p.threads) - scalars - 2048;
    p.buffers = static_cast<int>(std::min<size_t>(kMaxBuffers, std::max<size_t>(3, share / (static_cast<size_t>(p.per) * 16))));
    p.smem = static_cast<size_t>(p.buffers) * p.per * 16 + scalars;
    return p;
}

template <typename T, int THREADS, int GRAD> cudaError_t staged_config(const StagePlan &p, cudaLaunchConfig_t *cfg, cudaLaunchAttribute *at) {
    constexpr auto kernel = policy_staged_kernel<T, THREADS, GRAD>;
    cudaError_t e = allow_shared<kernel>(static_cast<int>(kSmBytes));
    if (e != cudaSuccess) return e;
    if (p.cs > 8 && (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    *cfg = {};
    cfg->gridDim = dim3(p.cs);
    cfg->blockDim = dim3(THREADS);
    cfg->dynamicSmemBytes = p.smem;
    at->id = cudaLaunchAttributeClusterDimension;
    at->val.clusterDim.x = p.cs;
    at->val.clusterDim.y = at->val.clusterDim.z = 1;
    cfg->attrs = at;
    cfg->numAttrs = 1;
    return cudaSuccess;
}

template <typename T, int THREADS, int GRAD> cudaError_t resident_clusters(StagePlan *p) {
    constexpr auto kernel = policy_staged_kernel<T, THREADS, GRAD>;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at;
    cudaError_t e = staged_config<T, THREADS, GRAD>(*p, &cfg, &at);
    if (e != cudaSuccess) return e;
    if (p->cs > 1) return cudaOccupancyMaxActiveClusters(&p->clusters, kernel, &cfg);
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&p->clusters, kernel, THREADS, p->smem);
    p->clusters *= sm_count_now();
    return e;
}

template <typename T, int THREADS, int GRAD> cudaError_t launch_staged(const PolicyArgs &a, const StagePlan &p, cudaStream_t s) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at;
    cudaError_t e = staged_config<T, THREADS, GRAD>(p, &cfg, &at);
    if (e != cudaSuccess) return e;
    Staging g;
    g.per = p.per;
    g.cs = p.cs;
    g.buffers = p.buffers;
    g.clusters = std::min<int64_t>(a.n, p.clusters);
    g.span = g.clusters * batch_rows(THREADS);
    // Masked rows cost a fraction of the others and come in no even order, so up to kRanked rows the live ones are dealt
    // out by rank: every CTA reads all weights and actions once (about 2 us for 8192 rows).  Beyond, and with short rows,
    // the strided deal evens out by itself.
    g.ranked = a.weights && THREADS == 512 && a.n <= std::min<int64_t>(kRanked, g.span);
    cfg.gridDim = dim3(static_cast<unsigned>(g.clusters * p.cs));
    cfg.stream = s;
    return cudaLaunchKernelEx(&cfg, policy_staged_kernel<T, THREADS, GRAD>, a, g);
}

// How rows are spread.  The time of a row is mostly latency (its loads, two reductions, its stores), so the rate goes
// with the rows that the device holds at once: of the fewest CTAs a row with slices of up to 512, 256 and 128
// threads, the one with the most clusters resident (8192 x 33000 bf16: 76, 101, 121 clusters take 308, 239 and
// 205 us; 1500 x 128001: 38 each, 133, 131, 138 us).  With fewer rows than that, a row takes as many CTAs as
// there are SMs for, in slices of 8 KB at least.  `found` is false where 16 CTAs do not hold a row: it is then read twice.
template <typename T, int GRAD> cudaError_t stage_plan(const PolicyArgs &a, StagePlan *plan, bool *found) {
    struct Known {
        int64_t granules;
        int device;
        StagePlan plan;
        bool found;
    };
    static thread_local Known last = {-1, -1, {}, false};
    const int64_t granules = row_granules(a, sizeof(T));
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    auto query = [](StagePlan *p) {
        return p->threads == 32 ? resident_clusters<T, 32, GRAD>(p) : p->threads == 64 ? resident_clusters<T, 64, GRAD>(p) : p->threads == 128 ? resident_clusters<T, 128, GRAD>(p)
               : p->threads == 256 ? resident_clusters<T, 256, GRAD>(p) : resident_clusters<T, 512, GRAD>(p);
    };
    if (last.granules != granules || last.device != dev) {
        Known k = {granules, dev, {}, false};
        for (int threads : {512, 256, 128}) {
            const int64_t cs = (granules + threads * kGranules - 1) / (threads * kGranules);
            if (cs > kMaxCluster) continue;
            StagePlan p = slice_plan(granules, static_cast<int>(cs));
            if ((e = query(&p)) != cudaSuccess) return e;
            if (p.clusters > k.plan.clusters) k.plan = p;
        }
        k.found = k.plan.clusters > 0;
        // more CTAs a row where that leaves as many clusters (512 x 200000 fp32: 13 a row 172 us, 16 a row 162)
        for (int cs = k.plan.cs + 1; k.found && k.plan.cs > 1 && cs <= kMaxCluster; ++cs) {
            StagePlan p = slice_plan(granules, cs);
            if ((e = query(&p)) != cudaSuccess) return e;
            if (p.clusters < k.plan.clusters) break;
            k.plan = p;
        }
        last = k;
    }
    *plan = last.plan;
    *found = last.found;
    if (!last.found || a.n * 2 > last.plan.clusters) return cudaSuccess;
    int cs = last.plan.cs;
    while (cs * 2 <= 8 && a.n * cs * 2 <= sm_count_now() && granules / cs >= 1024) cs *= 2;
    if (cs == last.plan.cs) return cudaSuccess;
    StagePlan p = slice_plan(granules, cs);
    if ((e = query(&p)) != cudaSuccess) return e;
    if (p.clusters > 0) *plan = p;
    return cudaSuccess;
}

template <typename T, int GRAD> cudaError_t launch_staged_rows(const PolicyArgs &a, cudaStream_t s, bool *done) {
    StagePlan p;
    cudaError_t e = stage_plan<T, GRAD>(a, &p, done);
    if (e != cudaSuccess || !*done) return e;
    return p.threads == 32 ? launch_staged<T, 32, GRAD>(a, p, s) : p.threads == 64 ? launch_staged<T, 64, GRAD>(a, p, s) : p.threads == 128 ? launch_staged<T, 128, GRAD>(a, p, s)
           : p.threads == 256 ? launch_staged<T, 256, GRAD>(a, p, s) : launch_staged<T, 512, GRAD>(a, p, s);
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
    bool done = false;
    cudaError_t e;
    if (dtype == CCQ_BF16)
        e = a.dlogits ? launch_staged_rows<__nv_bfloat16, 1>(a, s, &done) : launch_staged_rows<__nv_bfloat16, 0>(a, s, &done);
    else
        e = a.dlogits ? launch_staged_rows<float, 1>(a, s, &done) : launch_staged_rows<float, 0>(a, s, &done);
    if (e != cudaSuccess || done) return e;
    int b = access_bytes(static_cast<uintptr_t>(a.vocab) * es);
    b = row_access(a.logits, a.logits_stride, es, a.n, b);
    if (a.dlogits) b = row_access(a.dlogits, a.dlogits_stride, es, a.n, b);
    if (dtype == CCQ_BF16)
        return b == 16 ? launch_rows<__nv_bfloat16, 8>(a, s) : b >= 4 ? launch_rows<__nv_bfloat16, 2>(a, s)
                                                                      : launch_rows<__nv_bfloat16, 1>(a, s);
    return b == 16 ? launch_rows<float, 4>(a, s) : launch_rows<float, 1>(a, s);
}

void set_inverse(PolicyArgs *a) {
    const double inv = 1.0 / static_cast<double>(a->p.temperature);
    a->inv = static_cast<float>(inv);
    a->inv_lo = static_cast<float>(inv - static_cast<double>(a->inv));
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
    // (below 4.3e-39 log2(e) / temperature is infinite, and every row's largest logit 0 times that)
    if (!(temperature > 0.f) || temperature > 1e30f || !(kLog2e / temperature < INFINITY))
        return op_fail(CCQ_ERR_INVALID_ARG, "temperature=%g must be positive and finite, its reciprocal too",
                       static_cast<double>(temperature));
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
    if ((st = op_status_word(&a.status)) != CCQ_OK) return st;
    a.logits = logits; a.logits_stride = logits_stride; a.actions = actions; a.id_bytes = id_bytes;
    a.n = n; a.vocab = vocab;
    a.old_logp = old_logp; a.ref_logp = ref_logp; a.advantages = advantages; a.weights = weights;
    a.scale = kLog2e / a.p.temperature;
    set_inverse(&a);
    a.grad_mul = a.p.grad_scale / a.p.temperature;
    a.logp = logp; a.row_loss = static_cast<float *>(workspace);
    a.dlogits = dlogits; a.dlogits_stride = dlogits_stride;
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
    if ((st = op_status_word(&a.status)) != CCQ_OK) return st;
    a.logits = logits; a.logits_stride = logits_stride; a.actions = actions; a.id_bytes = id_bytes;
    a.n = n; a.vocab = vocab;
    a.p.temperature = temperature;
    a.scale = kLog2e / temperature;
    set_inverse(&a);
    a.logp = logp;
    a.score = 1;
    return op_cuda(launch_policy(a, dtype, static_cast<cudaStream_t>(stream)), "token log-probability launch");
}

}  // extern "C"

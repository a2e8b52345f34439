// ccq_norm.cu -- group norm of tokens, channels last, with an activation or a gate, and its gradients
// (ccq_ops.h).
//
// Both directions stream: the forward reads x (and the gate) and writes y, the backward reads x, the gate and
// dy and writes dx and dgate, each once.  A team of threads holds a (token, group)'s d channels in registers, K
// accesses of N elements each, so that the mean and the squared deviations from it (no cancellation for a group
// whose mean is large), and in the backward the two means of its formula, are sums over registers and a team:
//   s = act(gate), du = dy s, dgate = dy u act'(gate)      (no gate: du = dy act'(u))
//   dxh = du weight,  dx = rstd (dxh - mean(dxh) - xh mean(dxh xh))     (mean(dxh) = 0 with centered = 0)
//   dweight = sum over tokens of du xh,  dbias = sum over tokens of du
// A team keeps one group and walks over tokens, so that its weights, and the backward's partial sums of
// dweight and dbias, stay in registers too; the partial sums go to the workspace once and norm_param_kernel
// adds them in a fixed order.  A team is at most a warp where K accesses each suffice, else the
// whole CTA; groups beyond that (d > 4096) are walked in memory (norm_long_kernel).
// Measured, bf16 with a gate and groups of 128: forward of 32768 x 2048 64 us (6.3 TB/s, 93 % of the copy rate; HBM bounds
// it); backward of 16384 x 2048 62 us (5.4 TB/s, 80 %), of 65536 tokens 216 us (92 %): about 10 us of a call are its two
// launches, first loads and the parameters' partial sums, the rest HBM with the issue slots 62 % busy (41 instructions an
// element).  Groups of 33, one element an access: 31 and 26 %.
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
    int channels, groups, d, slots;
    int centered, act, param_bf16;
    float eps;
};

__device__ __forceinline__ float param_at(const void *p, int bf16, int i, float none) {
    if (!p) return none;
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ float sigmoid(float u) { return fast_rcp(1.f + fast_exp2(-1.4426950408889634f * u)); }

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

// Sum over the team: TEAM lanes of a warp, or (kWide) the CTA.  Every thread gets the same value.
constexpr int kWide = kThreads;
template <int TEAM> __device__ __forceinline__ float team_sum(float v, float *red) {
#pragma unroll
    for (int o = (TEAM < 32 ? TEAM : 32) >> 1; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if constexpr (TEAM > 32) {
        __syncthreads();  // the last sum's readers are done
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) v += red[w];
    }
    return v;
}

// Arithmetic on a thread's E channels, two at a time where E is even.
template <int E> __device__ __forceinline__ float v_sum(const float (&x)[E]) {
    if constexpr (E % 2) {
        return x[0];
    } else {
        uint64_t s = f2_make(x[0], x[1]);
#pragma unroll
        for (int i = 2; i < E; i += 2) s = f2_add(s, f2_make(x[i], x[i + 1]));
        const float2 t = f2_split(s);
        return t.x + t.y;
    }
}
template <int E> __device__ __forceinline__ float v_dot(const float (&x)[E], const float (&y)[E]) {
    if constexpr (E % 2) {
        return x[0] * y[0];
    } else {
        uint64_t s = f2_mul(f2_make(x[0], x[1]), f2_make(y[0], y[1]));
#pragma unroll
        for (int i = 2; i < E; i += 2) s = f2_fma(f2_make(x[i], x[i + 1]), f2_make(y[i], y[i + 1]), s);
        const float2 t = f2_split(s);
        return t.x + t.y;
    }
}
// d = x y + z, and its forms with a scalar
template <int E>
__device__ __forceinline__ void v_fma(float (&d)[E], const float (&x)[E], const float (&y)[E], const float (&z)[E]) {
    if constexpr (E % 2) {
        d[0] = x[0] * y[0] + z[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 t = f2_split(f2_fma(f2_make(x[i], x[i + 1]), f2_make(y[i], y[i + 1]), f2_make(z[i], z[i + 1])));
            d[i] = t.x;
            d[i + 1] = t.y;
        }
    }
}
template <int E> __device__ __forceinline__ void v_fma(float (&d)[E], const float (&x)[E], float y, const float (&z)[E]) {
    if constexpr (E % 2) {
        d[0] = x[0] * y + z[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 t = f2_split(f2_fma(f2_make(x[i], x[i + 1]), f2_make(y, y), f2_make(z[i], z[i + 1])));
            d[i] = t.x;
            d[i + 1] = t.y;
        }
    }
}
template <int E> __device__ __forceinline__ void v_mul(float (&d)[E], const float (&x)[E], const float (&y)[E]) {
    if constexpr (E % 2) {
        d[0] = x[0] * y[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 t = f2_split(f2_mul(f2_make(x[i], x[i + 1]), f2_make(y[i], y[i + 1])));
            d[i] = t.x;
            d[i + 1] = t.y;
        }
    }
}
template <int E> __device__ __forceinline__ void v_mul(float (&d)[E], const float (&x)[E], float y) {
    if constexpr (E % 2) {
        d[0] = x[0] * y;
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 t = f2_split(f2_mul(f2_make(x[i], x[i + 1]), f2_make(y, y)));
            d[i] = t.x;
            d[i + 1] = t.y;
        }
    }
}
template <int E> __device__ __forceinline__ void v_add(float (&d)[E], const float (&x)[E], const float (&y)[E]) {
    if constexpr (E % 2) {
        d[0] = x[0] + y[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 t = f2_split(f2_add(f2_make(x[i], x[i + 1]), f2_make(y[i], y[i + 1])));
            d[i] = t.x;
            d[i + 1] = t.y;
        }
    }
}
template <int E> __device__ __forceinline__ void v_add(float (&d)[E], const float (&x)[E], float y) {
    if constexpr (E % 2) {
        d[0] = x[0] + y;
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 t = f2_split(f2_add(f2_make(x[i], x[i + 1]), f2_make(y, y)));
            d[i] = t.x;
            d[i + 1] = t.y;
        }
    }
}

// act(u) of a thread's channels, and with SLOPE its derivative.  The activation is one for the launch: the branch
// stands outside the loops over channels (inside, it and the masks made 45 instructions an element of the forward).
template <int SLOPE, int E> __device__ __forceinline__ void v_act(int act, const float (&u)[E], float (&y)[E], float (&slope)[E]) {
    if (act == CCQ_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            y[i] = u[i];
            if constexpr (SLOPE) slope[i] = 1.f;
        }
        return;
    }
    float s[E];
    v_mul(s, u, -1.4426950408889634f);
#pragma unroll
    for (int i = 0; i < E; ++i) s[i] = fast_exp2(s[i]);
    v_add(s, s, 1.f);
#pragma unroll
    for (int i = 0; i < E; ++i) s[i] = fast_rcp(s[i]);
    if (act == CCQ_ACT_SILU) {
        v_mul(y, u, s);
        if constexpr (SLOPE) {  // s + u s (1 - s)
            float rest[E], one[E];
#pragma unroll
            for (int i = 0; i < E; ++i) one[i] = 1.f;
            v_fma(rest, s, -1.f, one);
            v_fma(slope, y, rest, s);
        }
    } else {
        if constexpr (SLOPE) {  // s (1 - s)
            float rest[E], one[E];
#pragma unroll
            for (int i = 0; i < E; ++i) one[i] = 1.f;
            v_fma(rest, s, -1.f, one);
            v_mul(slope, s, rest);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) y[i] = s[i];
    }
}

// x becomes (x - mu) / std, and 1 / std is returned; accesses past d hold zeros and stay zero (K accesses of N).
// Where every thread of a warp's team holds the same number of channels, its own mean and squared deviations are
// merged pairwise (the deviations of a pair of halves: the sum of theirs and n / 2 times the squared difference of their
// means), one chain of shuffles where the mean first and then the deviations takes two.  Neither loses
// digits to a large mean.
template <int TEAM, int N, int K>
__device__ __forceinline__ float normalise(float (&x)[N * K], int accesses, const NormArgs &a, float *red) {
    constexpr int E = N * K;
    const float inv_d = 1.f / static_cast<float>(a.d);
    float dev;
    if (TEAM <= 32 && a.centered && a.d == TEAM * E) {
        float mean = v_sum(x) * (1.f / E), y[E];
        v_add(y, x, -mean);
        dev = v_dot(y, y);
        float half = 0.5f * E;
#pragma unroll
        for (int o = 1; o < TEAM; o <<= 1) {
            const float om = __shfl_xor_sync(~0u, mean, o), od = __shfl_xor_sync(~0u, dev, o);
            const float diff = om - mean;
            mean = 0.5f * (mean + om);
            dev = (dev + od) + diff * diff * half;
            half *= 2.f;
        }
        v_add(x, x, -mean);
    } else {
        if (a.centered) {
            const float mu = team_sum<TEAM>(v_sum(x), red) * inv_d;
            if (accesses == K) {
                v_add(x, x, -mu);
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k)
                    if (k < accesses)
#pragma unroll
                        for (int e = 0; e < N; ++e) x[k * N + e] -= mu;
            }
        }
        dev = team_sum<TEAM>(v_dot(x, x), red);
    }
    const float rstd = rsqrtf(dev * inv_d + a.eps);
    v_mul(x, x, rstd);
    return rstd;
}

// Tokens whose operands are under way in shared memory (a thread copies its own accesses there, so no barrier is
// needed; bf16 elements one by one are below the copies' 4 bytes and are prefetched into registers, one token ahead).
template <typename T> constexpr int stages(int n, int k, int bwd) {
    const int bytes = n * static_cast<int>(sizeof(T)) * k * (bwd ? 3 : 2) * kThreads;
    return n * sizeof(T) < 4 ? 0 : bytes > 12288 ? 2 : 4;
}
template <typename T> constexpr int stage_bytes(int n, int k, int bwd) {
    return n * static_cast<int>(sizeof(T)) * k * (bwd ? 3 : 2) * kThreads;
}

// CTAs of norm_kernel on an SM, which bounds its registers and sets the grid.
constexpr int resident(int elems, int bwd) { return bwd ? (elems > 8 ? 1 : 2) : elems > 8 ? 2 : 4; }

// Forward (BWD = 0) and backward (BWD = 1) of groups held in registers: K accesses of N elements a thread.
template <typename T, int N, int K, int TEAM, int BWD>
__global__ void __launch_bounds__(kThreads, resident(N * K, BWD)) norm_kernel(NormArgs a) {
    constexpr int E = N * K;
    __shared__ float red[kThreads / 32];
    constexpr int kTeams = kThreads / TEAM;
    // the grid is at most a few CTAs an SM, or `unit` (of shape_of()) of them, at most one a group: below 2^24 x kThreads teams
    const uint32_t gt = blockIdx.x * kTeams + threadIdx.x / TEAM;
    const int l = threadIdx.x % TEAM;
    const int group = static_cast<int>(gt % static_cast<uint32_t>(a.groups));
    const int slot = static_cast<int>(gt / static_cast<uint32_t>(a.groups));
    const int base = group * a.d;
    int accesses = 0;  // of K, those below d
#pragma unroll
    for (int k = 0; k < K; ++k) accesses += (k * TEAM + l) * N < a.d;
    // this thread's first access of token t is at base + t rows (tokens and a row's bytes are below 2^31)
    const uint32_t row0 = static_cast<uint32_t>(slot), rows = static_cast<uint32_t>(a.slots);
    const int64_t c0 = base + l * N;
    const T *X = static_cast<const T *>(a.x) + c0, *G = static_cast<const T *>(a.gate) + c0;
    const T *DY = static_cast<const T *>(a.dy) + c0;
    T *Y = static_cast<T *>(a.y) + c0, *DG = static_cast<T *>(a.dgate) + c0;
    const uint32_t x_row = static_cast<uint32_t>(a.x_stride), g_row = static_cast<uint32_t>(a.gate_stride);
    const uint32_t dy_row = static_cast<uint32_t>(a.dy_stride), y_row = static_cast<uint32_t>(a.y_stride);
    const uint32_t dg_row = static_cast<uint32_t>(a.dgate_stride);
    auto row_at = [](auto *p, uint32_t t, uint32_t row) { return p + static_cast<uint64_t>(t) * row; };
    const bool gated = a.gate != nullptr;
    // tokens of this slot, and of the longest one: every thread of a warp walks as often, the sums are taken by
    // whole warps
    const int mine = slot < a.tokens ? static_cast<int>((a.tokens - slot + a.slots - 1) / a.slots) : 0;
    const int turns = static_cast<int>((a.tokens + a.slots - 1) / a.slots);
    constexpr int S = stages<T>(N, K, BWD);
    using P = Pack<T, N>;
    extern __shared__ __align__(16) uint8_t ring[];  // [S][operand][K][threads] accesses
    auto cell = [&](int stage, int operand, int k) {
        return reinterpret_cast<P *>(ring) + ((stage * (BWD ? 3 : 2) + operand) * K + k) * kThreads + threadIdx.x;
    };
    P px[K], pg[K], pd[K];
    auto fetch = [&](int turn) {
        const uint32_t t = row0 + turn * rows;
        if constexpr (S > 0) {
            if (turn < mine) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (k >= accesses) break;
                    copy_async<sizeof(P)>(cell(turn % S, 0, k), row_at(X, t, x_row) + k * TEAM * N);
                    if (gated) copy_async<sizeof(P)>(cell(turn % S, 1, k), row_at(G, t, g_row) + k * TEAM * N);
                    if constexpr (BWD)
                        copy_async<sizeof(P)>(cell(turn % S, 2, k), row_at(DY, t, dy_row) + k * TEAM * N);
                }
            }
            copy_commit();
        } else {
            // without conditions, so that all loads stay under way: past the end of the tokens the slot's first token (or the
            // first of all), past the group's end its last access, which take() drops
            const uint32_t from = turn < mine ? t : mine > 0 ? row0 : 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k < accesses ? k * TEAM : accesses > 0 ? (accesses - 1) * TEAM : -l) * N;
                px[k] = load_stream<T, N>(row_at(X, from, x_row) + c);
                if (gated) pg[k] = load_stream<T, N>(row_at(G, from, g_row) + c);
                if constexpr (BWD) pd[k] = load_stream<T, N>(row_at(DY, from, dy_row) + c);
            }
        }
    };
    if constexpr (S > 0) {
        // what is never copied (a token or access past the end, no gate) reads as zero
#pragma unroll
        for (int i = 0; i < S * (BWD ? 3 : 2); ++i)
#pragma unroll
            for (int k = 0; k < K; ++k) cell(0, i, k)->raw = {};
        for (int turn = 0; turn < S - 1; ++turn) fetch(turn);
    } else {
        fetch(0);
    }
    // (the first tokens' copies are under way by now)
    float w[E], b[E], dw[BWD ? E : 1], db[BWD ? E : 1];
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int c = (k * TEAM + l) * N + e, i = k * N + e;
            w[i] = c < a.d ? param_at(a.weight, a.param_bf16, base + c, 1.f) : 0.f;
            b[i] = c < a.d ? param_at(a.bias, a.param_bf16, base + c, 0.f) : 0.f;
            if constexpr (BWD) dw[i] = db[i] = 0.f;
        }
    }
    for (int turn = 0; turn < turns; ++turn) {
        const bool live = turn < mine;
        const uint32_t t = row0 + turn * rows;
        if constexpr (S > 0) {
            fetch(turn + S - 1);  // into the stage that the token before this one has left
            copy_wait<S - 1>();
        }
        // an operand's channels, taken from shared memory where they are needed
        auto take = [&](int operand, const P (&held)[K], float (&v)[E]) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float f[N];
                if constexpr (S > 0) {
                    const P p = *cell(turn % S, operand, k);
                    unpack(p, f);
                } else {
                    unpack(held[k], f);
                    if (k >= accesses) {
#pragma unroll
                        for (int e = 0; e < N; ++e) f[e] = 0.f;
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) v[k * N + e] = f[e];
            }
        };
        float x[E], g[E], dy[E];
        take(0, px, x);
        if constexpr (S == 0) {
            if (gated) take(1, pg, g);
            if constexpr (BWD) take(2, pd, dy);
        }
        if constexpr (S == 0) fetch(turn + 1);
        const float rstd = normalise<TEAM, N, K>(x, accesses, a, red);
        float u[E];
        v_fma(u, x, w, b);
        if (S > 0 && gated) take(1, pg, g);
        if constexpr (!BWD) {
            float none[E];
            if (gated) {
                v_act<0>(a.act, g, x, none);
                v_mul(x, x, u);
            } else {
                v_act<0>(a.act, u, x, none);
            }
        } else {
            // dy becomes du, then dxh = du w; g becomes dgate
            float y[E], slope[E];
            v_act<1>(a.act, gated ? g : u, y, slope);
            if (S > 0) take(2, pd, dy);
            if (gated) {
                v_mul(u, u, slope);
                v_mul(g, u, dy);
                v_mul(dy, dy, y);
            } else {
                v_mul(dy, dy, slope);
            }
            if (live) {  // (a token past the end has zeros, but 0 times an infinite 1 / std)
                v_fma(dw, dy, x, dw);
                v_add(db, db, dy);
            }
            v_mul(dy, dy, w);
            const float inv_d = 1.f / static_cast<float>(a.d);
            const float s1 = a.centered ? team_sum<TEAM>(v_sum(dy), red) * inv_d : 0.f;
            const float s2 = team_sum<TEAM>(v_dot(dy, x), red) * inv_d;
            float shift[E];
#pragma unroll
            for (int i = 0; i < E; ++i) shift[i] = -s1 * rstd;
            v_fma(x, x, -s2 * rstd, shift);
            v_fma(x, dy, rstd, x);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!live || k >= accesses) continue;
            float f[N];
            Pack<T, N> p;
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = x[k * N + e];
            pack(f, p);
            store_stream<T, N>(row_at(Y, t, y_row) + k * TEAM * N, p);
            if constexpr (BWD) {
                if (gated) {
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = g[k * N + e];
                    pack(f, p);
                    store_stream<T, N>(row_at(DG, t, dg_row) + k * TEAM * N, p);
                }
            }
        }
    }
    if constexpr (BWD) {
        if (!a.part) return;
        float *pw = a.part + static_cast<int64_t>(slot) * a.channels + base, *pb = pw + static_cast<int64_t>(a.slots) * a.channels;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TEAM + l) * N;
            if (c >= a.d) continue;
            if constexpr (N % 4 == 0) {  // d, and with it every group's first channel, is a multiple of N
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    const int i = k * N + e;
                    *reinterpret_cast<float4 *>(pw + c + e) = make_float4(dw[i], dw[i + 1], dw[i + 2], dw[i + 3]);
                    *reinterpret_cast<float4 *>(pb + c + e) = make_float4(db[i], db[i + 1], db[i + 2], db[i + 3]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    pw[c + e] = dw[k * N + e];
                    pb[c + e] = db[k * N + e];
                }
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
        pw = a.part + static_cast<int64_t>(slot) * a.channels + base;
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
            mu = team_sum<kWide>(s, red) * inv_d;
        }
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            const float v = to_f32(X[c]) - mu;
            q += v * v;
        }
        const float rstd = rsqrtf(team_sum<kWide>(q, red) * inv_d + a.eps);
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
        s1 = a.centered ? team_sum<kWide>(s1, red) * inv_d : 0.f;
        s2 = team_sum<kWide>(s2, red) * inv_d;
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

// dweight and dbias: 32 channels a CTA, the slots over 32 rows of threads (ten loads under way), then those 32 sums of
// a channel by a warp.
constexpr int kParamRows = 32;
__global__ void __launch_bounds__(32 * kParamRows) norm_param_kernel(const float *part, int slots, int channels,
                                                                     void *dweight, void *dbias, int param_bf16) {
    __shared__ float sums[kParamRows][33];
    grid_wait();
    const int which = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
    void *out = which ? dbias : dweight;
    if (!out) return;
    const float *p = part + static_cast<int64_t>(which) * slots * channels + min(c, channels - 1);
    float s = 0.f;
    for (int i0 = threadIdx.y; i0 < slots; i0 += 10 * kParamRows) {
        float v[10];
#pragma unroll
        for (int q = 0; q < 10; ++q) v[q] = p[static_cast<int64_t>(min(i0 + q * kParamRows, slots - 1)) * channels];
#pragma unroll
        for (int q = 0; q < 10; ++q) s += i0 + q * kParamRows < slots ? v[q] : 0.f;
    }
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    s = sums[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    const int mine = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x || mine >= channels) return;
    if (param_bf16) static_cast<__nv_bfloat16 *>(out)[mine] = __float2bfloat16_rn(s);
    else static_cast<float *>(out)[mine] = s;
}

// How the groups are spread over threads, and how many slots of tokens there are.
struct Shape {
    int n, k, team, slots;  // accesses of n elements, k a thread; team = 0: walked in memory
    unsigned grid;
};

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

Shape shape_of(int64_t tokens, int channels, int groups, int n, int bwd) {
    Shape s = {};
    const int d = channels / groups, packs = d / n, kmax = kMaxElems / n;
    s.n = n;
    s.k = 1;
    while (s.k < kmax && 32 * s.k < packs) s.k = n == 1 || n == 2 ? s.k * 4 : s.k * 2;
    s.k = std::min(s.k, kmax);
    if (32 * s.k >= packs) {
        s.team = s.k == 4 && n <= 2 ? (packs <= 64 ? 16 : 32) : s.k > 1 ? 32 : packs <= 1 ? 1 : packs <= 4 ? 4 : packs <= 8 ? 8 : packs <= 16 ? 16 : 32;
    } else if (kThreads * kmax >= packs) {
        s.k = kThreads >= packs ? 1 : kmax;
        s.team = kThreads;
    }
    const int teams = s.team ? kThreads / s.team : 1;  // a CTA's teams
    // a CTA count that is a multiple of `unit` gives every group the same number of teams
    const int unit = groups / gcd(groups, teams);
    // The forward takes four times the CTAs that fit at once, so that SMs that finish early take more (32768 x 2048
    // bf16, gated: 1 x 69.3, 2 x 66.7, 4 x 63.6, 8 x 67.6 us); the backward one wave, its slots' partial sums cost more
    // (16384 x 2048: 1 x 63.0, 2 x 67.9 us).  That is by the long walks: where a slot has few tokens four waves cost a
    // first fetch each (gated bf16 after an L2 flush, 1 and 4 waves: 4096 x 16 x 128 17.1 and 21.2 us, 20000 x 1 x 2048 49.8 and
    // 56.0, 65536 x 4 x 64 25.2 and 27.3, 32768 x 16 x 128 76.4 and 70.3).
    const int64_t most = static_cast<int64_t>(sm_count_now()) * (s.team ? resident(n * s.k, bwd) * (bwd ? 1 : 4) : 4);
    const int64_t want = std::min<int64_t>(most, (tokens * groups + teams - 1) / teams);
    const int64_t grid = std::max<int64_t>(1, want / unit) * unit;
    s.grid = static_cast<unsigned>(grid);
    s.slots = static_cast<int>(grid * teams / groups);
    return s;
}

template <typename T, int N, int K, int TEAM, int BWD> cudaError_t launch_team(const NormArgs &a, const Shape &sh, cudaStream_t s) {
    constexpr int smem = stages<T>(N, K, BWD) * stage_bytes<T>(N, K, BWD);
    if constexpr (smem > 40960) {
        cudaError_t e = allow_shared<norm_kernel<T, N, K, TEAM, BWD>>(smem);
        if (e != cudaSuccess) return e;
    }
    norm_kernel<T, N, K, TEAM, BWD><<<sh.grid, kThreads, smem, s>>>(a);
    return cudaGetLastError();
}

// With one access a thread the team is as small as holds the group; with more it is a warp, or the CTA.
template <typename T, int N, int K, int BWD> cudaError_t launch_one(const NormArgs &a, const Shape &sh, cudaStream_t s) {
    if constexpr (K == 1) {
        switch (sh.team) {
            case 1: return launch_team<T, N, K, 1, BWD>(a, sh, s);
            case 4: return launch_team<T, N, K, 4, BWD>(a, sh, s);
            case 8: return launch_team<T, N, K, 8, BWD>(a, sh, s);
            case 16: return launch_team<T, N, K, 16, BWD>(a, sh, s);
        }
    }
    if constexpr (K == 4 && N <= 2)
        if (sh.team == 16) return launch_team<T, N, K, 16, BWD>(a, sh, s);
    if constexpr (K == 1 || N * K == kMaxElems)
        if (sh.team == kWide) return launch_team<T, N, K, kWide, BWD>(a, sh, s);
    return launch_team<T, N, K, 32, BWD>(a, sh, s);
}

template <typename T, int BWD> cudaError_t launch_norm(NormArgs a, const Shape &sh, cudaStream_t s) {
    a.slots = sh.slots;
    if (!sh.team) {
        norm_long_kernel<T, BWD><<<sh.grid, kThreads, 0, s>>>(a);
        return cudaGetLastError();
    }
    if constexpr (sizeof(T) == 2) {
        if (sh.n == 8)
            return sh.k == 1 ? launch_one<T, 8, 1, BWD>(a, sh, s) : launch_one<T, 8, 2, BWD>(a, sh, s);
        if (sh.n == 4)
            return sh.k == 1   ? launch_one<T, 4, 1, BWD>(a, sh, s)
                   : sh.k == 2 ? launch_one<T, 4, 2, BWD>(a, sh, s)
                               : launch_one<T, 4, 4, BWD>(a, sh, s);
        if (sh.n == 2)
            return sh.k == 1   ? launch_one<T, 2, 1, BWD>(a, sh, s)
                   : sh.k == 4 ? launch_one<T, 2, 4, BWD>(a, sh, s)
                               : launch_one<T, 2, 8, BWD>(a, sh, s);
    } else if (sh.n == 4) {
        return sh.k == 1   ? launch_one<T, 4, 1, BWD>(a, sh, s)
               : sh.k == 2 ? launch_one<T, 4, 2, BWD>(a, sh, s)
                           : launch_one<T, 4, 4, BWD>(a, sh, s);
    }
    return sh.k == 1   ? launch_one<T, 1, 1, BWD>(a, sh, s)
           : sh.k == 4 ? launch_one<T, 1, 4, BWD>(a, sh, s)
                       : launch_one<T, 1, 16, BWD>(a, sh, s);
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
    if (channels > (1 << 24)) return op_fail(CCQ_ERR_UNSUPPORTED, "channels=%d: supported up to 2^24", channels);
    if (tokens > 0x7fffffff)
        return op_fail(CCQ_ERR_UNSUPPORTED, "tokens=%lld: supported below 2^31", static_cast<long long>(tokens));
    return CCQ_OK;
}

// One [tokens, channels] operand; `least` shrinks to its access width.
ccq_status check_operand(const char *name, const void *p, int64_t stride, int64_t tokens, int channels, int es, int *least) {
    if (tokens > 1 && stride < channels)
        return op_fail(CCQ_ERR_INVALID_ARG, "%s: row stride %lld is below the %d channels", name,
                       static_cast<long long>(stride), channels);
    if (tokens > 1 && stride > 0x7fffffff)
        return op_fail(CCQ_ERR_UNSUPPORTED, "%s: row stride %lld: supported below 2^31", name, static_cast<long long>(stride));
    *least = row_access(p, stride, es, tokens, *least);
    return op_pointer(name, p, es);
}

// Elements of the widest access with its kernels: 16 bytes, 8 or 4 of bf16, or one element.
int access_elems(int bytes, int es) { return bytes == 16 ? 16 / es : es == 2 ? bytes / 2 : 1; }

ccq_status check_param(const char *name, const void *p, ccq_dtype dt) {
    return p ? op_pointer(name, p, dtype_bytes(dt)) : CCQ_OK;
}

// The most slots any access width gives: bounds the partial sums.
size_t bwd_workspace(int64_t tokens, int channels, int groups, int es) {
    int slots = 1;
    for (int n : {16 / es, 4, 2, 1})
        if ((channels / groups) % n == 0) slots = std::max(slots, shape_of(tokens, channels, groups, n, 1).slots);
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
    const Shape sh = shape_of(tokens, channels, groups, access_elems(b, es), 0);
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
    const Shape sh = shape_of(tokens, channels, groups, access_elems(b, es), 1);
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

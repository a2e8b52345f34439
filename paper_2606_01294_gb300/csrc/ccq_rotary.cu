// ccq_rotary.cu -- rotation of the heads of queries and keys by their positions (ccq_ops.h).
//
// The pair (a, b) of a token at position p turns by p f_i radians: a' = m (a cos - b sin), b' = m (a sin + b cos).
// Angles are kept as 64-bit fractions of a turn: F_i = f_i 2^64 / (2 pi) mod 2^64 and p F_i mod 2^64 in integers, where F_i is within
// 3 units of 2^-64 turns; the top 32 bits become the argument of sincospif, rounded to fp32.  Positions of more than 32 bits and
// frequencies from 2 on, which lose more, take 128-bit fractions (far_angle).  (The same in 64-bit floating point, at this GPU's rate
// for it, would take a fifth of the prefill's time.)  A CTA computes the cosines and sines of its tokens once for all heads.
// Bound by HBM, every element read once and written once: 8 x 4096 tokens of 16 + 16 heads of 128 in bf16 80 us, 6.7 TB/s, a copy's
// rate.  A decode's 256 tokens take 3 us, a launch.
#include <algorithm>

#include "ccq_ops.cuh"

namespace ccq {
namespace {

constexpr int kThreads = 256;
constexpr int kMostAngles = 2048;  // of a CTA: 16 KB of shared memory

struct RotaryTensor {
    const void *x;
    void *y;
    int64_t xb, xt, xh, yb, yt, yh;
    int heads;
};

// n / d for 0 <= n < 2^31 as a product: with 2^s the first power of two from d on and m = floor(2^32 (2^s - d) / d) + 1,
// n / d = (floor(m n / 2^32) + n) / 2^s (Granlund and Montgomery's method).
struct Divisor {
    uint32_t m, s;
    Divisor() = default;
    explicit Divisor(uint32_t d) {
        s = 0;
        while ((1ull << s) < d) ++s;
        m = static_cast<uint32_t>(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ int operator()(int n) const { return static_cast<int>((__umulhi(m, n) + static_cast<uint32_t>(n)) >> s); }
};

struct RotaryArgs {
    RotaryTensor t[2];
    int heads;             // of both tensors
    int64_t tokens, T;     // B * T, T
    int width, part;
    const void *positions;
    int position_bytes;
    const double *freqs;
    float amplitude;
    int inverse;
    int tile;              // tokens of a CTA
    int turned, items;     // a head's rotated items, and with those that are copied
    Divisor by_token, by_items, by_T, by_half;  // (a division by a number that is known here is several dozen instructions, by T
                                                // in 64 bits a hundred: they took a third of the 3 x 3001 tokens' time)
};

// f 2^64 / (2 pi) mod 2^64 within 3 units, from the bits of f, for |f| < 2.
__device__ __forceinline__ uint64_t turns_of(double f) {
    constexpr uint64_t kInvTwoPi = 2935890503282001226ull;  // 2^64 / (2 pi)
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(f));
    const int e = static_cast<int>((bits >> 52) & 0x7ff);
    uint64_t m = bits & 0xfffffffffffffull;
    m = e ? m | (1ull << 52) : 0;  // (a subnormal frequency turns by nothing)
    const uint64_t hi = __umul64hi(m << 11, kInvTwoPi);  // f = (m << 11) 2^(e - 1086): F = hi 2^(e - 1022)
    const int s = e - 1022;
    const uint64_t F = s <= -64 ? 0 : s > 0 ? hi << s : hi >> -s;
    return bits >> 63 ? 0 - F : F;
}

// 1 / (2 pi), 64 bits a word, the first behind the point.
__device__ constexpr uint64_t kInverseTurn[19] = {
    0x28be60db9391054aull, 0x7f09d5f47d4d3770ull, 0x36d8a5664f10e410ull, 0x7f9458eaf7aef158ull, 0x6dc91b8e909374b8ull,
    0x01924bba82746487ull, 0x3f877ac72c4a69cfull, 0xba208d7d4baed121ull, 0x3a671c09ad17df90ull, 0x4e64758e60d4ce7dull,
    0x272117e2ef7e4a0eull, 0xc7fe25fff7816603ull, 0xfbcbc462d6829b47ull, 0xdb4d9fb3c9f2c26dull, 0xd3d18fd9a797fa8bull,
    0x5d49eeb1faf97c5eull, 0xcf41ce7de294a4baull, 0x9afed7ec47e35742ull, 0x1580cc11bf1edaeaull};

// The angle p f, in units of 2^-32 turns, for any p and any finite f = +-m 2^k: m, of 53 bits, times the 192 bits of 1 / (2 pi) from
// the first whose product is no whole turn (Payne and Hanek's reduction) leaves 128 bits behind the point, and |p| takes 63 of them.
__device__ __noinline__ int32_t far_angle(int64_t p, double f) {
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(f));
    const int e = static_cast<int>((bits >> 52) & 0x7ff), k = e - 1075;
    if (k <= -192) return 0;  // (below 2^-75 turns at any p)
    const uint64_t m = (bits & 0xfffffffffffffull) | (1ull << 52);
    const int first = k >> 6, shift = k & 63;
    auto word = [](int j) { return j < 0 ? 0 : kInverseTurn[j]; };
    uint64_t x[3];
#pragma unroll
    for (int i = 0; i < 3; ++i)
        x[i] = shift ? word(first + i) << shift | word(first + i + 1) >> (64 - shift) : word(first + i);
    const uint64_t mid = m * x[1], lo = mid + __umul64hi(m, x[2]), hi = m * x[0] + __umul64hi(m, x[1]) + (lo < mid);
    const uint64_t n = p < 0 ? 0 - static_cast<uint64_t>(p) : static_cast<uint64_t>(p);
    const uint64_t turn = n * hi + __umul64hi(n, lo);
    return static_cast<int32_t>(((bits >> 63) != (p < 0) ? 0 - turn : turn) >> 32);
}

// The angle of every day, by one product: within 2^-30 of a turn, as 3 units of F times |p| <= 2^31 and the cut at 32 bits are.
__device__ __forceinline__ int32_t angle_of(int64_t p, double f) {
    const int exponent = __double2hiint(f) >> 20 & 0x7ff;  // (no comparison in 64 bits)
    if (p != static_cast<int32_t>(p) || exponent > 1023) return far_angle(p, f);
    return static_cast<int32_t>((static_cast<uint64_t>(p) * turns_of(f)) >> 32);
}

// N elements an access; PAIR: the two halves of N pairs as an access each (N = 1 interleaved: its two elements), else an
// access holds N / 2 pairs side by side.
template <typename T, int N, bool PAIR, bool INTER>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryArgs a) {
    // [tile][part / 2]: cos, sin; of the pairs of an access two by two, those of neighbouring accesses side by side, so that a warp's
    // reads do not meet in a bank (8 x 4096 tokens, 32 heads of 128 in bf16: 90 us where they do, 86 so, both before the divisions went)
    extern __shared__ __align__(16) float2 turn[];
    constexpr int kPairs = PAIR ? N : N / 2;  // of an access
    const int half = a.part / 2, across = half / kPairs;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.tile;
    const int tokens = static_cast<int>(min(static_cast<int64_t>(a.tile), a.tokens - first));
    for (int j = threadIdx.x; j < tokens * half; j += kThreads) {
        const int t = a.by_half(j), i = j - t * half;
        const double f = a.freqs[i];
        const int32_t angle = angle_of(load_index(a.positions, a.position_bytes, first + t), f);
        float s, c;
        sincospif(static_cast<float>(angle) * 0x1p-31f, &s, &c);
        if (!isfinite(f)) s = c = __int_as_float(0x7fffffff);
        const int e = i % kPairs, place = kPairs == 1 ? i : (e / 2 * across + i / kPairs) * 2 + e % 2;
        turn[t * half + place] = make_float2(c * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
    }
    __syncthreads();
    const int per_token = a.heads * a.items;
    constexpr int K = N * sizeof(T) <= 4 || !PAIR ? 4 : 2;  // items at once
    const int total = tokens * per_token;
    for (int j0 = threadIdx.x; j0 < total; j0 += K * kThreads) {
        Pack<T, N> u[K], w[K];
        T *out[K];
        int angle[K], second[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int j = min(j0 + k * kThreads, total - 1);  // (without conditions, so that all loads stay under way)
            const int t = a.by_token(j), r = j - t * per_token;
            int h = a.by_items(r);
            const int c = r - h * a.items;
            const bool key = h >= a.t[0].heads;
            const RotaryTensor &x = a.t[key];
            if (key) h -= a.t[0].heads;
            const int row = static_cast<int>(first) + t;  // (below 2^31)
            const int64_t b = a.by_T(row), at = row - b * a.T;
            int64_t from = b * x.xb + at * x.xt + h * x.xh, to = b * x.yb + at * x.yt + h * x.yh;
            int lo;
            second[k] = 0;
            if (c < a.turned) {
                lo = PAIR && INTER ? 2 * c : c * N;
                if (PAIR) second[k] = INTER ? 1 : half;
                angle[k] = t * half + (kPairs == 1 ? c : 2 * c);
            } else {
                lo = a.part + (c - a.turned) * N;
                angle[k] = -1;
            }
            const T *src = static_cast<const T *>(x.x) + from + lo;
            u[k] = load_stream<T, N>(src);
            if (PAIR) w[k] = load_stream<T, N>(src + second[k]);
            out[k] = static_cast<T *>(x.y) + to + lo;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (j0 + k * kThreads >= total) continue;
            if (angle[k] < 0) {
                store_stream<T, N>(out[k], u[k]);
                continue;
            }
            float p[N], q[N];
            unpack(u[k], p);
            if constexpr (PAIR) unpack(w[k], q);
            auto rotate = [](float &x, float &y, float c, float s) {
                const float r = x * c - y * s;
                y = x * s + y * c;
                x = r;
            };
            if constexpr (kPairs == 1) {
                const float2 cs = turn[angle[k]];
                if constexpr (PAIR)
                    rotate(p[0], q[0], cs.x, cs.y);
                else
                    rotate(p[0], p[1], cs.x, cs.y);
            } else {
#pragma unroll
                for (int e = 0; e < kPairs; e += 2) {
                    const float4 cs = *reinterpret_cast<const float4 *>(&turn[angle[k] + e * across]);
                    if constexpr (PAIR) {
                        rotate(p[e], q[e], cs.x, cs.y);
                        rotate(p[e + 1], q[e + 1], cs.z, cs.w);
                    } else {
                        rotate(p[2 * e], p[2 * e + 1], cs.x, cs.y);
                        rotate(p[2 * e + 2], p[2 * e + 3], cs.z, cs.w);
                    }
                }
            }
            if constexpr (PAIR) {
                pack(q, w[k]);
                store_stream<T, N>(out[k] + second[k], w[k]);
            }
            pack(p, u[k]);
            store_stream<T, N>(out[k], u[k]);
        }
    }
}

template <typename T, int N, bool PAIR, bool INTER>
cudaError_t launch(RotaryArgs &a, bool in_place, cudaStream_t s) {
    a.turned = PAIR ? a.part / 2 / N : a.part / N;
    a.items = a.turned + (in_place ? 0 : (a.width - a.part) / N);
    const int half = a.part / 2;
    // tokens of a CTA: four accesses a thread where the tokens fill the GPU (3 x 3001 tokens interleaved 14 us, 16.5 with six, 22 with
    // two; 8 x 4096 80, 81, 79), one token (latency) where they do not
    const int per_token = a.heads * a.items;
    const int64_t fill = a.tokens / (8 * sm_count_now());
    const int want = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(fill, (4 * kThreads) / per_token)));
    a.tile = std::max(1, std::min(want, kMostAngles / half));
    const int64_t grid = (a.tokens + a.tile - 1) / a.tile;
    a.by_token = Divisor(per_token);
    a.by_items = Divisor(a.items);
    a.by_T = Divisor(static_cast<uint32_t>(a.T));
    a.by_half = Divisor(half);
    rotary_kernel<T, N, PAIR, INTER><<<static_cast<unsigned>(grid), kThreads, a.tile * half * sizeof(float2), s>>>(a);
    return cudaGetLastError();
}

template <typename T> cudaError_t by_access(RotaryArgs &a, int bytes, bool interleaved, bool in_place, cudaStream_t s) {
    const int n = bytes / static_cast<int>(sizeof(T));
    constexpr int N16 = 16 / sizeof(T), N8 = 8 / sizeof(T), N4 = 4 / sizeof(T);
    if (interleaved) {
        if (n >= N16) return launch<T, N16, false, true>(a, in_place, s);
        if (n >= 2 && n >= N8) return launch<T, N8, false, true>(a, in_place, s);
        if constexpr (N4 >= 2)
            if (n >= N4) return launch<T, N4, false, true>(a, in_place, s);
        return launch<T, 1, true, true>(a, in_place, s);
    }
    if (n >= N16) return launch<T, N16, true, false>(a, in_place, s);
    if (n >= N8) return launch<T, N8, true, false>(a, in_place, s);
    if constexpr (N4 >= 2)
        if (n >= N4) return launch<T, N4, true, false>(a, in_place, s);
    return launch<T, 1, true, false>(a, in_place, s);
}

}  // namespace
}  // namespace ccq

using namespace ccq;

extern "C" {

ccq_status ccq_rotary(const ccq_heads *x, const ccq_heads *y, int count, ccq_dtype dtype, int64_t B, int64_t T, int width,
                      int part, const void *positions, int position_bytes, const double *freqs, float amplitude,
                      int interleaved, int inverse, void *stream) {
    if (count < 1 || count > 2) return op_fail(CCQ_ERR_INVALID_ARG, "count=%d: one or two tensors", count);
    if (!x || !y) return op_fail(CCQ_ERR_INVALID_ARG, "x or y is NULL");
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", static_cast<int>(dtype));
    ccq_status st = check_tokens(B, T);
    if (st != CCQ_OK) return st;
    if (width < 2 || width > 65536 || part < 2 || part > width || part % 2)
        return op_fail(CCQ_ERR_INVALID_ARG, "head width %d with %d rotated: an even part from 2 to the width (at most 65536)",
                       width, part);
    if (part / 2 > kMostAngles) return op_fail(CCQ_ERR_UNSUPPORTED, "at most %d rotated channels a head", 2 * kMostAngles);
    if (position_bytes != 4 && position_bytes != 8)
        return op_fail(CCQ_ERR_INVALID_ARG, "position_bytes=%d: 4 or 8", position_bytes);
    if (!isfinite(amplitude)) return op_fail(CCQ_ERR_INVALID_ARG, "amplitude is not finite");
    const int elem = dtype_bytes(dtype);
    RotaryArgs a = {};
    // elements of an access: what the pairs' places, the strides and the addresses of all tensors divide by
    int bytes = access_bytes(static_cast<uintptr_t>(width) * elem);
    bytes = access_bytes(static_cast<uintptr_t>(interleaved ? part : part / 2) * elem, bytes);
    bytes = access_bytes(static_cast<uintptr_t>(width - part) * elem, bytes);
    bool in_place = true;
    int64_t heads = 0;
    for (int i = 0; i < count; ++i) {
        const char *names[2][2] = {{"x[0]", "y[0]"}, {"x[1]", "y[1]"}};
        if ((st = check_heads(names[i][0], x[i], dtype, B, T, width, false)) != CCQ_OK) return st;
        if ((st = check_heads(names[i][1], y[i], dtype, B, T, width, true)) != CCQ_OK) return st;
        if (x[i].heads != y[i].heads) return op_fail(CCQ_ERR_INVALID_ARG, "x[%d] and y[%d] differ in heads", i, i);
        bytes = heads_access(x[i], elem, B, T, heads_access(y[i], elem, B, T, bytes));
        a.t[i] = {x[i].p, y[i].p, x[i].batch, x[i].token, x[i].head, y[i].batch, y[i].token, y[i].head,
                  static_cast<int>(x[i].heads)};
        in_place = in_place && x[i].p == y[i].p && (B <= 1 || x[i].batch == y[i].batch) &&
                   (T <= 1 || x[i].token == y[i].token) && (x[i].heads <= 1 || x[i].head == y[i].head);
        heads += x[i].heads;
    }
    if (heads * width > (1 << 24)) return op_fail(CCQ_ERR_UNSUPPORTED, "at most 2^24 channels a token");
    if (B * T == 0) return CCQ_OK;
    if ((st = op_pointer("positions", positions, position_bytes)) != CCQ_OK) return st;
    if ((st = op_pointer("freqs", freqs, 8)) != CCQ_OK) return st;
    for (int i = 0; i < count; ++i) {
        if (x[i].p == y[i].p && ((B > 1 && x[i].batch != y[i].batch) || (T > 1 && x[i].token != y[i].token) ||
                                 (x[i].heads > 1 && x[i].head != y[i].head)))
            return op_fail(CCQ_ERR_INVALID_ARG, "y[%d] is x[%d] with other strides", i, i);
        if (count == 2 && (y[i].p == x[1 - i].p || y[0].p == y[1].p))
            return op_fail(CCQ_ERR_INVALID_ARG, "y[%d] is %s[%d]", i, y[i].p == x[1 - i].p ? "x" : "y", 1 - i);
    }
    const char *xs[2] = {"x[0]", "x[1]"}, *ys[2] = {"y[0]", "y[1]"};
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < count; ++j) {
            if ((i != j || x[i].p != y[i].p) && (st = check_apart(ys[i], y[i], xs[j], x[j], elem, B, T, width)) != CCQ_OK) return st;
            if (i < j && (st = check_apart(ys[j], y[j], ys[i], y[i], elem, B, T, width)) != CCQ_OK) return st;
        }
    a.heads = static_cast<int>(heads);
    a.tokens = B * T;
    a.T = T;
    a.width = width;
    a.part = part;
    a.positions = positions;
    a.position_bytes = position_bytes;
    a.freqs = freqs;
    a.amplitude = amplitude;
    a.inverse = inverse != 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return op_cuda(dtype == CCQ_BF16 ? by_access<__nv_bfloat16>(a, bytes, interleaved != 0, in_place, s)
                                     : by_access<float>(a, bytes, interleaved != 0, in_place, s),
                   "rotary launch");
}

}  // extern "C"

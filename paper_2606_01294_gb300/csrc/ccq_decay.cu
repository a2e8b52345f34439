// ccq_decay.cu -- linear attention with a decay for each head in fp32 arithmetic, for any type and alignment, and the
// entry points (ccq_ops.h).  ccq_decay.cuh says how one pass serves the forward and the gradients.
//
// decay_block_kernel: a CTA walks the tokens of one (sequence, head, segment) in blocks of 32 with a slice of 32 columns of
// the state, in fp32 on the CUDA cores:
//   P = Q K^T (32 x 32), masked and times g^|i - j|;  O = P V + diag(g^..) Q S;  S = g^n S + K^T diag(g^..) V.
// Half of the threads have the state and what is read from it (Q S), the others P and P V: between its two barriers a block is one chain
// of either.  32 tokens cost 32 d (32 + 2 * 32) + 20 * 32 * 32 multiply-adds a CTA, of which P, formed whole and again by each slice, is
// a third.
// Aligned fp32 operands of the next block are copied while this one is computed.
// Bound by what a thread loads from shared memory (32 words a cycle for an SM that multiplies 128): so Q K^T and Q S are 4 x 8 a
// thread over a quarter of d, summed by shuffles, and P V reads four columns of P at a time.  What is left is instructions: Q S and the
// state's increment are multiplied in pairs (531 -> 496 us; Q K^T in pairs, with twice the sums, is slower for d = 64).  8 x 1000
// tokens of 16 heads of 128 in fp32: 482 us (797 with 2 x 4 a thread and one group), 8 x 1000 x 16 x 64 159 (287), 4 x 777 of 4 heads of
// 64 in 7 segments 29 (49).
// Slices of 32 columns rather than whole heads, so that few heads still reach many SMs.
#include <algorithm>
#include <cmath>

#include "ccq_decay.cuh"

namespace ccq {
namespace {

constexpr int kC = 32;        // tokens of a block
constexpr int kN = 32;        // columns of a CTA
constexpr int kThreads = 256;
constexpr int kPad = 4;
constexpr int kRowPad = 16;   // of q and k: the two rows that eight lanes read lie in different halves of the banks

template <int D, int BUFFERS> struct BlockShared {
    struct {
        float q[kC][D + kRowPad], k[kC][D + kRowPad], v[kC][kN + kPad];
    } in[BUFFERS];
    float p[kC][kN + kPad], o[kC][kN + kPad];
    float s[D][kN];       // chunks of four columns swizzled by the row, as state_chunk() says
    float power[kC + 1];  // g^n
    float2 keep[2];       // g^32 and g^n of the ragged block, as two floats
};

// Where the four columns 4 c .. of a row of the state lie in its row: lanes that read rows four apart meet in no bank.
__device__ __forceinline__ int state_chunk(int row, int c) { return 4 * (c ^ (2 * (row >> 2 & 3))); }

// Sums of 4 x 8 over four neighbouring lanes; lane l keeps columns 2 l and 2 l + 1.
__device__ __forceinline__ void sum_lanes(float (&x)[4][8], int l, float (&y)[4][2]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            x[r][c] = (l & 2 ? x[r][c + 4] : x[r][c]) + __shfl_xor_sync(0xffffffffu, l & 2 ? x[r][c] : x[r][c + 4], 2);
#pragma unroll
        for (int c = 0; c < 2; ++c)
            y[r][c] = (l & 1 ? x[r][c + 2] : x[r][c]) + __shfl_xor_sync(0xffffffffu, l & 1 ? x[r][c] : x[r][c + 2], 1);
    }
}

// Rows begin .. begin + n of a head (of `width` channels from column c0) to shared memory, zeros up to kC.
template <typename T, int W, int STRIDE>
__device__ __forceinline__ void load_rows(float (*dst)[STRIDE], const DecayView &x, int64_t b, int64_t begin, int n, int h,
                                          int c0, bool vec) {
    const T *src = static_cast<const T *>(x.p) + b * x.batch + begin * x.token + (h / x.share) * x.head + c0;
    if (vec) {
        constexpr int N = 16 / sizeof(T);
        for (int j = threadIdx.x; j < kC * W / N; j += kThreads) {
            const int r = j / (W / N), c = (j % (W / N)) * N;
            float f[N];
            if (r < n) {
                const Pack<T, N> p = load_plain<T, N>(src + r * x.token + c);
                unpack(p, f);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) f[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < N; e += 4)
                *reinterpret_cast<float4 *>(&dst[r][c + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
        }
    } else {
        for (int j = threadIdx.x; j < kC * W; j += kThreads) {
            const int r = j / W, c = j % W;
            dst[r][c] = r < n ? to_f32(src[r * x.token + c]) : 0.f;
        }
    }
}

// The same by asynchronous copies (aligned fp32).
template <int W, int STRIDE>
__device__ __forceinline__ void copy_rows(float (*dst)[STRIDE], const DecayView &x, int64_t b, int64_t begin, int n, int h,
                                          int c0) {
    const float *src = static_cast<const float *>(x.p) + b * x.batch + begin * x.token + (h / x.share) * x.head + c0;
    for (int j = threadIdx.x; j < kC * W / 4; j += kThreads) {
        const int r = j / (W / 4), c = (j % (W / 4)) * 4;
        if (r < n)
            copy_async<16>(&dst[r][c], src + r * x.token + c);
        else
            *reinterpret_cast<float4 *>(&dst[r][c]) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
}

// ASYNC: fp32 operands on 16-byte boundaries, copied a block ahead.
template <typename T, int D, bool ASYNC, bool PARTS>
__global__ void __launch_bounds__(kThreads, 2) decay_block_kernel(const DecayArgs a) {
    constexpr int kBuffers = ASYNC ? 2 : 1;
    if (PARTS) grid_release();  // (the launch after this one forms its tables and loads its first blocks meanwhile)
    extern __shared__ float4 shared_raw[];
    BlockShared<D, kBuffers> &sh = *reinterpret_cast<BlockShared<D, kBuffers> *>(shared_raw);
    constexpr int kSlices = D / kN;
    constexpr int R = PARTS ? D / 32 : D / 16;  // state rows of a thread: R x 4 of its slice
    constexpr int kWide = R % 4 ? 2 : 4;
    int64_t x = blockIdx.x;
    const int slice = static_cast<int>(x % kSlices);
    x /= kSlices;
    const int nseg = PARTS ? a.segments - 1 : a.segments;
    const int segment = static_cast<int>(x % nseg);
    x /= nseg;
    const int h = static_cast<int>(x % a.H);
    x /= a.H;
    const int sequence = decay_longest_first(a, static_cast<int>(x % a.sequences), reinterpret_cast<int *>(shared_raw));
    const DecayPass &ps = a.pass[x / a.sequences];
    const int tid = threadIdx.x, tx = tid % 8;
    const bool states = PARTS || tid >= kThreads / 2;  // these threads have the state and what is read from it, the others P and O
    const int ty = (PARTS ? tid : tid % (kThreads / 2)) / 8;
    // of the two products over d: rows 4 ti .., eight columns by tj, and of each 16 channels the four from 4 tk
    const int tk = tid % 4, tj = tid / 4 % 4, ti = tid % (kThreads / 2) / 16;
    const int c0 = slice * kN;
    const bool down = ps.descending != 0;

    const DecaySpan span = decay_span(a, sequence);
    const int64_t blocks = (span.length + kC - 1) / kC, per = (blocks + a.segments - 1) / a.segments;
    const int64_t first = min(per * segment, blocks), last = min(first + per, blocks);
    const DecayLog l2 = decay_log2(a.log_decay, h);
    const int ragged = static_cast<int>(span.length - (blocks - 1) * kC);  // tokens of the sequence's last block
    if (tid <= kC) sh.power[tid] = decay_power(l2, tid);
    if (tid >= kThreads - 2) sh.keep[tid - (kThreads - 2)] = decay_keep(l2, tid == kThreads - 2 ? kC : ragged);

    // the factors of the segments before this one, as two floats (up to 64 products; where P will lie)
    float2 *seg_keep = reinterpret_cast<float2 *>(&sh.p[0][0]);
    auto segment_tokens = [&](int g) {
        const int64_t lo = min(per * g, blocks), hi = min(per * (g + 1), blocks);
        return lo < hi ? static_cast<int>((hi - lo) * kC - ((down ? lo == 0 : hi == blocks) ? blocks * kC - span.length : 0)) : 0;
    };
    if (!PARTS && a.segments > 1 && tid < segment) seg_keep[tid] = decay_keep(l2, segment_tokens(tid));

    if (a.cu || (!PARTS && a.segments > 1)) __syncthreads();  // (the ranks' place becomes the first block's)
    // tokens of block j in the pass's order: the ragged block is the sequence's last
    auto block_begin = [&](int64_t j) { return (down ? blocks - 1 - j : j) * kC; };

    auto tokens_of = [&](int64_t begin) { return static_cast<int>(min(static_cast<int64_t>(kC), span.length - begin)); };
    auto copy = [&](int64_t j) {
        if constexpr (ASYNC) {
            const int64_t begin = block_begin(j);
            const int n = tokens_of(begin);
            auto &to = sh.in[j & 1];
            copy_rows<D>(to.k, ps.k, span.b, span.begin + begin, n, h, 0);
            copy_rows<kN>(to.v, ps.v, span.b, span.begin + begin, n, h, c0);
            if (!PARTS) copy_rows<D>(to.q, ps.q, span.b, span.begin + begin, n, h, 0);
            copy_commit();
        }
    };
    if (first < last) copy(first);
    if (a.segments > 1 && !PARTS) grid_wait();  // (the segments' parts)

    // ---- the state at the segment's start; this thread's rows R ty .. and columns 4 tx ..
    float S[R][4];
    {
        const int64_t at = (static_cast<int64_t>(sequence) * a.H + h) * D * D;
        auto add = [&](const float *m, bool transposed, float2 keep) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int row = R * ty + r, col = c0 + 4 * tx + c;
                    const float f = m[transposed ? col * D + row : row * D + col];
                    S[r][c] = keep.x == 0.f ? f : fmaf(S[r][c], keep.x, fmaf(S[r][c], keep.y, f));
                }
            }
        };
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) S[r][c] = 0.f;
        if (!states) {
        } else if (a.segments == 1 || (PARTS && segment == 0)) {
            if (ps.state_in) add(ps.state_in + at, ps.transposed, make_float2(0.f, 0.f));
            if (PARTS) {
                float *to = a.parts + decay_part(a, ps.kind, sequence, h, 0);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    *reinterpret_cast<float4 *>(to + (R * ty + r) * D + c0 + 4 * tx) =
                        make_float4(S[r][0], S[r][1], S[r][2], S[r][3]);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) S[r][c] = 0.f;
            }
        } else if (!PARTS) {
            for (int g = 0; g <= segment; ++g)
                add(a.parts + decay_part(a, ps.kind, sequence, h, g), ps.parts_transposed, g ? seg_keep[g - 1] : make_float2(0.f, 0.f));
        }
    }

    for (int64_t j = first; j < last; ++j) {
        const int64_t begin = block_begin(j);
        const int n = tokens_of(begin);
        auto &in = sh.in[ASYNC ? j & 1 : 0];
        // (all have read the last block: the barrier at its end, or no block was)
        if constexpr (ASYNC) {
            if (j + 1 < last) {
                copy(j + 1);
                copy_wait<1>();
            } else {
                copy_wait<0>();
            }
        } else {
            load_rows<T, D>(in.k, ps.k, span.b, span.begin + begin, n, h, 0, a.vec);
            load_rows<T, kN>(in.v, ps.v, span.b, span.begin + begin, n, h, c0, a.vec);
            if (!PARTS) load_rows<T, D>(in.q, ps.q, span.b, span.begin + begin, n, h, 0, a.vec);
        }
        if (!PARTS && states) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                *reinterpret_cast<float4 *>(&sh.s[R * ty + r][state_chunk(R * ty + r, tx)]) =
                    make_float4(S[r][0], S[r][1], S[r][2], S[r][3]);
        }
        __syncthreads();
        float o[2][4] = {};  // rows 2 ty, 2 ty + 1, columns 4 tx .. 4 tx + 3
        if (states) {
            if constexpr (!PARTS) {
                // diag(g^..) Q S: columns 4 tj .. and 16 + 4 tj ..
                float x[4][8], y[4][2];
                uint64_t x2[4][4] = {};
#pragma unroll 2
                for (int e = 4 * tk; e < D; e += 16) {
                    float4 qv[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) qv[r] = *reinterpret_cast<const float4 *>(&in.q[4 * ti + r][e]);
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const float4 s0 = *reinterpret_cast<const float4 *>(&sh.s[e + f][state_chunk(e, tj)]),
                                     s1 = *reinterpret_cast<const float4 *>(&sh.s[e + f][state_chunk(e, tj + 4)]);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float w = f == 0 ? qv[r].x : f == 1 ? qv[r].y : f == 2 ? qv[r].z : qv[r].w;
                            const uint64_t ww = f2_make(w, w);
                            x2[r][0] = f2_fma(ww, f2_make(s0.x, s0.y), x2[r][0]);
                            x2[r][1] = f2_fma(ww, f2_make(s0.z, s0.w), x2[r][1]);
                            x2[r][2] = f2_fma(ww, f2_make(s1.x, s1.y), x2[r][2]);
                            x2[r][3] = f2_fma(ww, f2_make(s1.z, s1.w), x2[r][3]);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float2 f = f2_split(x2[r][c]);
                        x[r][2 * c] = f.x;
                        x[r][2 * c + 1] = f.y;
                    }
                sum_lanes(x, tk, y);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 4 * ti + r, m = down ? n - 1 - i : i + 1;
                    const float f = m >= 0 ? sh.power[m] * ps.s_scale : 0.f;
                    *reinterpret_cast<float2 *>(&sh.o[i][16 * (tk >> 1) + 4 * tj + 2 * (tk & 1)]) = make_float2(y[r][0] * f, y[r][1] * f);
                }
            }
            // S = g^n S + K^T diag(k_scale g^..) V, rows R ty .., columns 4 tx ..
            const float2 keep = sh.keep[n < kC];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) S[r][c] = fmaf(S[r][c], keep.x, S[r][c] * keep.y);
#pragma unroll 1
            for (int j0 = 0; j0 < n; j0 += 4) {  // (rows past n are zeros)
                float4 vv[4];
                Pack<float, kWide> kv[4][R / kWide];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    vv[e] = *reinterpret_cast<const float4 *>(&in.v[j0 + e][4 * tx]);
#pragma unroll
                    for (int r = 0; r < R / kWide; ++r) kv[e][r] = load_plain<float, kWide>(&in.k[j0 + e][R * ty + kWide * r]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float u = sh.power[max(down ? j0 + e + 1 : n - 1 - j0 - e, 0)] * ps.k_scale;
                    vv[e].x *= u;
                    vv[e].y *= u;
                    vv[e].z *= u;
                    vv[e].w *= u;
#pragma unroll
                    for (int r = 0; r < R / kWide; ++r) {
                        float kk[kWide];
                        unpack(kv[e][r], kk);
#pragma unroll
                        for (int f = 0; f < kWide; ++f) {
                            float *row = S[kWide * r + f];
                            const uint64_t k2 = f2_make(kk[f], kk[f]);
                            const float2 a2 = f2_split(f2_fma(k2, f2_make(vv[e].x, vv[e].y), f2_make(row[0], row[1])));
                            const float2 b2 = f2_split(f2_fma(k2, f2_make(vv[e].z, vv[e].w), f2_make(row[2], row[3])));
                            row[0] = a2.x;
                            row[1] = a2.y;
                            row[2] = b2.x;
                            row[3] = b2.y;
                        }
                    }
                }
            }
        } else if constexpr (!PARTS) {
            // P: columns tj + 4 c
            float x[4][8] = {}, y[4][2];
#pragma unroll 2
            for (int e = 4 * tk; e < D; e += 16) {
                float4 qv[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) qv[r] = *reinterpret_cast<const float4 *>(&in.q[4 * ti + r][e]);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float4 kv = *reinterpret_cast<const float4 *>(&in.k[tj + 4 * c][e]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r][c] += qv[r].x * kv.x + qv[r].y * kv.y + qv[r].z * kv.z + qv[r].w * kv.w;
                }
            }
            sum_lanes(x, tk, y);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int i = 4 * ti + r, jj = tj + 4 * (2 * tk + c), gap = down ? jj - i : i - jj;
                    sh.p[i][jj] = gap >= 0 ? y[r][c] * (sh.power[gap] * ps.p_scale) : 0.f;
                }
            }
            __syncwarp();  // (a warp reads the rows that it has written)
            // O = P V, four columns of P at a time: those that all of the warp's eight rows keep, then those on the diagonal, where a
            // value that is not finite must not reach the rows before it
            const int row0 = ty / 4 * 8;
            auto four = [&](int j0, bool diagonal) {
                float4 vv[4], pv[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) pv[r] = *reinterpret_cast<const float4 *>(&sh.p[2 * ty + r][j0]);
#pragma unroll
                for (int e = 0; e < 4; ++e) vv[e] = *reinterpret_cast<const float4 *>(&in.v[j0 + e][4 * tx]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const bool kept = !diagonal || (down ? j0 + e >= 2 * ty + r : j0 + e <= 2 * ty + r);
                        const float w = e == 0 ? pv[r].x : e == 1 ? pv[r].y : e == 2 ? pv[r].z : pv[r].w;
                        o[r][0] = kept ? o[r][0] + w * vv[e].x : o[r][0];
                        o[r][1] = kept ? o[r][1] + w * vv[e].y : o[r][1];
                        o[r][2] = kept ? o[r][2] + w * vv[e].z : o[r][2];
                        o[r][3] = kept ? o[r][3] + w * vv[e].w : o[r][3];
                    }
                }
            };
#pragma unroll 1
            for (int j0 = down ? row0 + 8 : 0; j0 < (down ? n : row0); j0 += 4) four(j0, false);
#pragma unroll 1
            for (int j0 = row0; j0 < row0 + 8; j0 += 4) four(j0, true);
        }
        __syncthreads();
        if constexpr (!PARTS) {
            if (states) continue;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = 2 * ty + r;
                if (i >= n) continue;
                const float4 f = *reinterpret_cast<const float4 *>(&sh.o[i][4 * tx]);
                o[r][0] += f.x;
                o[r][1] += f.y;
                o[r][2] += f.z;
                o[r][3] += f.w;
                const int64_t at = span.b * ps.o_batch + (span.begin + begin + i) * ps.o_token + h * ps.o_head + c0 + 4 * tx;
                if (ps.o_fp32) {
                    float *to_p = static_cast<float *>(ps.o) + at;
                    *reinterpret_cast<float4 *>(to_p) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
                } else {
                    T *to_p = static_cast<T *>(ps.o) + at;
                    if (a.vec) {
                        Pack<T, 4> u;
                        pack(o[r], u);
                        store_stream<T, 4>(to_p, u);
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) to_p[c] = from_f32<T>(o[r][c]);
                    }
                }
            }
        }
    }
    float *to = nullptr;
    if (PARTS)
        to = a.parts + decay_part(a, ps.kind, sequence, h, segment + 1);
    else if (ps.state_out && segment == a.segments - 1)
        to = ps.state_out + (static_cast<int64_t>(sequence) * a.H + h) * D * D;
    if (to && states) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            *reinterpret_cast<float4 *>(to + (R * ty + r) * D + c0 + 4 * tx) = make_float4(S[r][0], S[r][1], S[r][2], S[r][3]);
    }
}

template <typename T, int D, bool ASYNC> cudaError_t launch_blocks(const DecayArgs &a, cudaStream_t s) {
    constexpr int kBytes = sizeof(BlockShared<D, ASYNC ? 2 : 1>);
    const int64_t grid = static_cast<int64_t>(D / kN) * (a.parts_only ? a.segments - 1 : a.segments) * a.H * a.sequences * a.passes;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    const unsigned ctas = static_cast<unsigned>(grid);
    cudaError_t e;
    if (a.parts_only) {
        if ((e = allow_shared<decay_block_kernel<T, D, ASYNC, true>>(kBytes)) != cudaSuccess) return e;
        decay_block_kernel<T, D, ASYNC, true><<<ctas, kThreads, kBytes, s>>>(a);
        return cudaGetLastError();
    }
    if ((e = allow_shared<decay_block_kernel<T, D, ASYNC, false>>(kBytes)) != cudaSuccess) return e;
    if (a.segments > 1) return launch_after(decay_block_kernel<T, D, ASYNC, false>, ctas, kThreads, kBytes, s, a);
    decay_block_kernel<T, D, ASYNC, false><<<ctas, kThreads, kBytes, s>>>(a);
    return cudaGetLastError();
}

// ---------------------------------------------------------------- gradients of shared heads

struct SumArgs {
    void *out[3];
    int64_t token[3], batch[3], head[3];
    const float *parts[3];  // [rows][H][d]
    int share[3];
    int count;
    int H, d;
    int64_t rows, T;
};

// out[row, head, c] = sum over the heads that read it, in ascending order; one thread four channels.  Bound by HBM and L2: parts of
// 3 x 1501 tokens, 16 heads of 64 twice (37 MB) 10 us.
template <typename Type> __global__ void __launch_bounds__(256) decay_sum_kernel(const SumArgs a, int vec) {
    const int which = blockIdx.x % a.count;
    const unsigned shift = a.d == 128 ? 5 : 4;  // four channels a thread
    const unsigned share = a.share[which], per_row = (a.H / share) << shift, rows = max(256 / per_row, 1u), blocks = gridDim.x / a.count;
    const unsigned own = threadIdx.x / per_row, r0 = threadIdx.x - own * per_row, T = static_cast<unsigned>(a.T);
    grid_wait();  // (the passes' parts)
    if (own >= rows) return;
    for (int64_t at = static_cast<int64_t>(blockIdx.x / a.count) * rows + own; at < a.rows; at += static_cast<int64_t>(blocks) * rows) {
        const unsigned row = static_cast<unsigned>(at), b = row / T, t = row - b * T;
        for (unsigned r = r0; r < per_row; r += 256) {
            const unsigned h = r >> shift, c = (r - (h << shift)) * 4;
            const float *src = a.parts[which] + (at * a.H + static_cast<int64_t>(h) * share) * a.d + c;
            float f[4] = {};
#pragma unroll 4
            for (unsigned g = 0; g < share; ++g) {
                const float4 u = __ldcs(reinterpret_cast<const float4 *>(src + static_cast<int64_t>(g) * a.d));
                f[0] += u.x;
                f[1] += u.y;
                f[2] += u.z;
                f[3] += u.w;
            }
            Type *to = static_cast<Type *>(a.out[which]) + b * a.batch[which] + t * a.token[which] + h * a.head[which] + c;
            if (vec) {
                Pack<Type, 4> p;
                pack(f, p);
                store_stream<Type, 4>(to, p);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] = from_f32<Type>(f[e]);
            }
        }
    }
}

// ---------------------------------------------------------------- the calls

// Segments of each sequence, by a count of what a launch takes: rounds of resident CTAs times the blocks of a CTA, for the
// passes and, with more than one segment, for the states before them (`kinds`, all segments but the last).  A block's times
// are those measured with the GPU full.  What is not counted: the adding of earlier segments' states, one after another (64 KB of each for
// d = 128), which few heads with dozens of segments feel.  1 x 16 x 20480 x 128 bf16: 482 us whole, 122 in 9 segments; the gradients of
// 4 x 16 x 4096 x 128: 197 whole, 249 in 2 each, 171 with 40 of 192 passes in 2; 1 x 8 x 4000 x 128 fp32: 162 in 9.
struct Cost {
    int block;           // tokens
    double main, parts;  // microseconds a block
    double launch;
    int resident;        // CTAs the GPU holds
};

struct Plan {
    int segments = 1, pairs = 0, pass = 0;  // DecayArgs' segments, split_pairs and split_pass
};

Plan plan_segments(int64_t B, int64_t T, int H, int d, int64_t num_seqs, ccq_dtype dtype, int passes) {
    Plan best;
    if (num_seqs < 1 || B * T < 1) return best;
    const bool cores = dtype == CCQ_BF16;
    const Cost c = cores ? Cost{128, d == 128 ? 3.45 : 2.4, d == 128 ? 4.0 : 2.8, 6.0, sm_count_now()}
                         : Cost{kC, d == 128 ? 8.7 : 5.1, d == 128 ? 3.5 : 2.5, 6.0, 2 * sm_count_now()};
    const int64_t ctas = num_seqs * H * (cores ? 1 : d / kN), blocks = (B * T / num_seqs + c.block - 1) / c.block;
    const int64_t kinds = passes > 1 ? 2 : 1;
    auto rounds = [&](int64_t n) { return static_cast<double>((n + c.resident - 1) / c.resident); };
    double least = rounds(ctas * passes) * static_cast<double>(blocks) * c.main;
    for (int s = 2; s <= 64 && s <= blocks / 2; ++s) {
        const double per = static_cast<double>((blocks + s - 1) / s);
        const double t = rounds(ctas * passes * s) * per * c.main + rounds(ctas * kinds * (s - 1)) * per * c.parts + c.launch;
        if (t < least) {
            least = t;
            best = {s, static_cast<int>(num_seqs * H), 0};
        }
    }
    // Full rounds of whole passes, and of what is left over (of the gradients dk and dv, which start from the same states) segments
    // that fit beside their parts' launch into the last one.  Packed sequences are not of one length, and their short ones come last.
    const int64_t all = ctas * passes, full = all / c.resident, rest = all % c.resident;
    const int64_t split = passes > 1 ? passes - 1 : 1, pairs = (rest + split - 1) / split;
    if (cores && num_seqs == B && full && rest)
        for (int s = 2; s <= 64 && s <= blocks / 2 && pairs * (split * s + s - 1) <= c.resident; ++s) {
            const double per = static_cast<double>((blocks + s - 1) / s);
            const double t = static_cast<double>(full * blocks) * c.main + per * std::max(c.main, c.parts) + c.launch;
            if (t < least) {
                least = t;
                best = {s, static_cast<int>(pairs), static_cast<int>(passes - split)};
            }
        }
    return best;
}

size_t parts_bytes(const Plan &p, int d, int kinds) {
    return p.segments > 1 ? static_cast<size_t>(kinds) * p.pairs * p.segments * d * d * 4 : 0;
}

ccq_status check_sizes(int64_t B, int64_t T, int H, int d, int64_t num_seqs) {
    ccq_status st = check_tokens(B, T);
    if (st != CCQ_OK) return st;
    if (H < 1 || H > (1 << 20)) return op_fail(CCQ_ERR_INVALID_ARG, "bad sizes: H=%d", H);
    if (d != 64 && d != 128) return op_fail(CCQ_ERR_UNSUPPORTED, "d=%d: 64 or 128", d);
    if (num_seqs < 0 || num_seqs > (1 << 24) || num_seqs * H > (1 << 24))
        return op_fail(CCQ_ERR_UNSUPPORTED, "%lld sequences of %d heads: at most 2^24 of both",
                       static_cast<long long>(num_seqs), H);
    return CCQ_OK;
}

ccq_status check_shared(const char *name, const ccq_heads &x, ccq_dtype dtype, int64_t B, int64_t T, int H, int d, bool apart) {
    ccq_status st = check_heads(name, x, dtype, B, T, d, apart);
    if (st != CCQ_OK) return st;
    if (x.heads > H || H % x.heads)
        return op_fail(CCQ_ERR_INVALID_ARG, "%s has %lld heads, no divisor of %d", name, static_cast<long long>(x.heads), H);
    return CCQ_OK;
}

ccq_status check_common(ccq_dtype dtype, const float *log_decay, float scale, int64_t B, int64_t T, int H, int d,
                        const void *cu, int cu_bytes, int64_t num_seqs) {
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", static_cast<int>(dtype));
    ccq_status st = check_sizes(B, T, H, d, num_seqs);
    if (st != CCQ_OK) return st;
    if (!std::isfinite(scale)) return op_fail(CCQ_ERR_INVALID_ARG, "scale is not finite");
    if ((st = op_pointer("log_decay", log_decay, 4)) != CCQ_OK) return st;
    if (!cu) {
        if (num_seqs != B) return op_fail(CCQ_ERR_INVALID_ARG, "num_seqs=%lld without cu, B=%lld",
                                          static_cast<long long>(num_seqs), static_cast<long long>(B));
        return CCQ_OK;
    }
    if (B != 1) return op_fail(CCQ_ERR_INVALID_ARG, "cu with B=%lld: packed sequences have B = 1", static_cast<long long>(B));
    if (cu_bytes != 4 && cu_bytes != 8) return op_fail(CCQ_ERR_INVALID_ARG, "cu_bytes=%d: 4 or 8", cu_bytes);
    return op_pointer("cu", cu, cu_bytes);
}

// States that a call reads while it writes others: apart, or (with `same`) the same ones.
ccq_status check_states_apart(const char *in, const float *read, const char *out, const float *written, size_t bytes, bool same) {
    if (!read || !written || !bytes || (same && read == written)) return CCQ_OK;
    const uintptr_t r = reinterpret_cast<uintptr_t>(read), w = reinterpret_cast<uintptr_t>(written);
    return (r < w ? w - r : r - w) < bytes ? op_fail(CCQ_ERR_INVALID_ARG, "%s overlaps %s", out, in) : CCQ_OK;
}

ccq_status check_state(const char *name, const float *p) {
    return p ? op_pointer(name, p, 16) : CCQ_OK;
}

// (one head's values as all heads, by a stride of 0, are one shared head)
DecayView view_of(const ccq_heads &x, int H) {
    return {x.p, x.batch, x.token, x.head, static_cast<int>(x.head == 0 ? H : H / x.heads)};
}

// Whether a tensor can be loaded in tiles: its batch rows and tokens do not step by nothing, and no step has 2^40 bytes.
bool steps(const ccq_heads &x, int64_t B, int64_t T) {
    constexpr int64_t most = (1LL << 39) - 1;
    return (B <= 1 || (x.batch > 0 && x.batch <= most)) && (T <= 1 || (x.token > 0 && x.token <= most)) &&
           (x.heads <= 1 || x.head <= most);
}

// parts_mask: the passes whose states the segments start from.
ccq_status run_passes(DecayArgs &a, const Plan &plan, ccq_dtype dtype, bool cores, int64_t B, unsigned parts_mask, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    a.segments = 1;
    if (cores || plan.pairs == a.sequences * a.H) {  // (decay_block_kernel splits all or nothing)
        a.segments = plan.segments;
        a.split_pairs = plan.pairs;
        a.split_pass = plan.pass;
    }
    for (int i = 0; i < a.passes; ++i) a.exact_state |= a.pass[i].state_out != nullptr;
    auto run = [&](const DecayArgs &x) { return cores ? launch_decay_chunks(x, B, s) : launch_decay_blocks(x, dtype, s); };
    if (a.segments > 1) {
        DecayArgs p = a;
        p.parts_only = 1;
        p.passes = 0;
        for (int i = 0; i < a.passes; ++i)
            if (parts_mask >> i & 1 && i >= a.split_pass) p.pass[p.passes++] = a.pass[i];
        e = run(p);
    }
    if (e == cudaSuccess) e = run(a);
    return op_cuda(e, "decayed attention launch");
}

}  // namespace

cudaError_t launch_decay_blocks(const DecayArgs &a, ccq_dtype dtype, cudaStream_t s) {
    if (dtype == CCQ_BF16)
        return a.d == 128 ? launch_blocks<__nv_bfloat16, 128, false>(a, s) : launch_blocks<__nv_bfloat16, 64, false>(a, s);
    if (!a.vec) return a.d == 128 ? launch_blocks<float, 128, false>(a, s) : launch_blocks<float, 64, false>(a, s);
    return a.d == 128 ? launch_blocks<float, 128, true>(a, s) : launch_blocks<float, 64, true>(a, s);
}

}  // namespace ccq

using namespace ccq;

extern "C" {

ccq_status ccq_decay_attention_workspace_size(int64_t B, int64_t T, int H, int d, int64_t num_seqs, ccq_dtype dtype,
                                              size_t *bytes) {
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", static_cast<int>(dtype));
    ccq_status st = check_sizes(B, T, H, d, num_seqs);
    if (st != CCQ_OK) return st;
    if (!bytes) return op_fail(CCQ_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = parts_bytes(plan_segments(B, T, H, d, num_seqs, dtype, 1), d, 1);
    return CCQ_OK;
}

ccq_status ccq_decay_attention(const ccq_heads *q, const ccq_heads *k, const ccq_heads *v, ccq_dtype dtype,
                               const float *log_decay, float scale, const float *S0, const ccq_heads *o, float *ST, int64_t B,
                               int64_t T, int H, int d, const void *cu, int cu_bytes, int64_t num_seqs, void *workspace,
                               size_t workspace_bytes, void *stream) {
    if (!q || !k || !v || !o) return op_fail(CCQ_ERR_INVALID_ARG, "q, k, v or o is NULL");
    ccq_status st = check_common(dtype, log_decay, scale, B, T, H, d, cu, cu_bytes, num_seqs);
    if (st != CCQ_OK) return st;
    const ccq_heads *in[3] = {q, k, v};
    const char *names[3] = {"q", "k", "v"};
    int access = 16;
    for (int i = 0; i < 3; ++i) {
        if ((st = check_shared(names[i], *in[i], dtype, B, T, H, d, false)) != CCQ_OK) return st;
        access = heads_access(*in[i], dtype_bytes(dtype), B, T, access);
    }
    if ((st = check_shared("o", *o, dtype, B, T, H, d, true)) != CCQ_OK) return st;
    if (o->heads != H) return op_fail(CCQ_ERR_INVALID_ARG, "o has %lld heads, expected %d", static_cast<long long>(o->heads), H);
    for (int i = 0; i < 3 && B * T; ++i)
        if (in[i]->p == o->p) return op_fail(CCQ_ERR_INVALID_ARG, "o is %s: other tokens still read it", names[i]);
    access = heads_access(*o, dtype_bytes(dtype), B, T, access);
    if ((st = check_state("S0", S0)) != CCQ_OK) return st;
    if ((st = check_state("ST", ST)) != CCQ_OK) return st;
    DecayArgs a = {};
    const Plan plan = plan_segments(B, T, H, d, num_seqs, dtype, 1);
    const size_t need = parts_bytes(plan, d, 1);
    if (need && (st = op_pointer("workspace", workspace, 16)) != CCQ_OK) return st;
    if (workspace_bytes < need)
        return op_fail(CCQ_ERR_INVALID_ARG, "workspace of %zu bytes, needs %zu", workspace_bytes, need);
    for (int i = 0; i < 3; ++i)
        if ((st = check_apart("o", *o, names[i], *in[i], dtype_bytes(dtype), B, T, d)) != CCQ_OK) return st;
    const size_t state_bytes = static_cast<size_t>(num_seqs) * H * d * d * 4;
    if ((st = check_states_apart("S0", S0, "ST", ST, state_bytes, true)) != CCQ_OK) return st;
    if (num_seqs == 0) return CCQ_OK;
    if ((st = op_status_word(&a.status)) != CCQ_OK) return st;
    a.passes = 1;
    DecayPass &p = a.pass[0];
    p.q = view_of(*q, H);
    p.k = view_of(*k, H);
    p.v = view_of(*v, H);
    p.o = o->p;
    p.o_batch = o->batch;
    p.o_token = o->token;
    p.o_head = o->head;
    p.state_in = S0;
    p.state_out = ST;
    p.p_scale = p.s_scale = scale;
    p.k_scale = 1.f;
    a.H = H;
    a.d = d;
    a.T = T;
    a.sequences = static_cast<int>(num_seqs);
    a.log_decay = log_decay;
    a.cu = cu;
    a.cu_bytes = cu_bytes;
    a.parts = static_cast<float *>(workspace);
    a.vec = access == 16;
    const bool cores = dtype == CCQ_BF16 && a.vec && B * T > 0 && steps(*q, B, T) && steps(*k, B, T) && steps(*v, B, T) &&
                       steps(*o, B, T);
    return run_passes(a, plan, dtype, cores, B, 1u, static_cast<cudaStream_t>(stream));
}

ccq_status ccq_decay_attention_bwd_workspace_size(int64_t B, int64_t T, int H, int q_heads, int k_heads, int v_heads, int d,
                                                  int64_t num_seqs, ccq_dtype dtype, size_t *bytes) {
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", static_cast<int>(dtype));
    ccq_status st = check_sizes(B, T, H, d, num_seqs);
    if (st != CCQ_OK) return st;
    size_t shared = 0;
    for (int heads : {q_heads, k_heads, v_heads}) {
        if (heads < 1 || heads > H || H % heads) return op_fail(CCQ_ERR_INVALID_ARG, "%d heads, no divisor of %d", heads, H);
        shared += heads < H;
    }
    if (!bytes) return op_fail(CCQ_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = parts_bytes(plan_segments(B, T, H, d, num_seqs, dtype, 3), d, 2) +
             shared * static_cast<size_t>(B * T) * H * d * 4;
    return CCQ_OK;
}

ccq_status ccq_decay_attention_bwd(const ccq_heads *q, const ccq_heads *k, const ccq_heads *v, ccq_dtype dtype,
                                   const float *log_decay, float scale, const float *S0, const ccq_heads *dout,
                                   const float *dST, const ccq_heads *dq, const ccq_heads *dk, const ccq_heads *dv, float *dS0,
                                   int64_t B, int64_t T, int H, int d, const void *cu, int cu_bytes, int64_t num_seqs,
                                   void *workspace, size_t workspace_bytes, void *stream) {
    if (!q || !k || !v || !dout || !dq || !dk || !dv) return op_fail(CCQ_ERR_INVALID_ARG, "a tensor of heads is NULL");
    ccq_status st = check_common(dtype, log_decay, scale, B, T, H, d, cu, cu_bytes, num_seqs);
    if (st != CCQ_OK) return st;
    const ccq_heads *in[4] = {q, k, v, dout}, *out[3] = {dq, dk, dv};
    const char *names[4] = {"q", "k", "v", "dout"}, *outs[3] = {"dq", "dk", "dv"};
    int access = 16, access_out = 16;
    size_t shared = 0;
    for (int i = 0; i < 4; ++i) {
        if ((st = check_shared(names[i], *in[i], dtype, B, T, H, d, false)) != CCQ_OK) return st;
        access = heads_access(*in[i], dtype_bytes(dtype), B, T, access);
    }
    if (dout->heads != H)
        return op_fail(CCQ_ERR_INVALID_ARG, "dout has %lld heads, expected %d", static_cast<long long>(dout->heads), H);
    for (int i = 0; i < 3; ++i) {
        if ((st = check_shared(outs[i], *out[i], dtype, B, T, H, d, true)) != CCQ_OK) return st;
        if (out[i]->heads != in[i]->heads)
            return op_fail(CCQ_ERR_INVALID_ARG, "%s has %lld heads, %s %lld", outs[i], static_cast<long long>(out[i]->heads),
                           names[i], static_cast<long long>(in[i]->heads));
        for (int j = 0; j < 4 && B * T; ++j)
            if (in[j]->p == out[i]->p) return op_fail(CCQ_ERR_INVALID_ARG, "%s is %s: other passes still read it", outs[i], names[j]);
        access_out = heads_access(*out[i], dtype_bytes(dtype), B, T, access_out);
        shared += out[i]->heads < H;
    }
    if ((st = check_state("S0", S0)) != CCQ_OK) return st;
    if ((st = check_state("dST", dST)) != CCQ_OK) return st;
    if ((st = check_state("dS0", dS0)) != CCQ_OK) return st;
    if (dS0 && dS0 == dST) return op_fail(CCQ_ERR_INVALID_ARG, "dS0 is dST: both are in use at once");
    DecayArgs a = {};
    const Plan plan = plan_segments(B, T, H, d, num_seqs, dtype, 3);
    const size_t states = parts_bytes(plan, d, 2);
    const size_t rows = static_cast<size_t>(B * T) * H * d * 4, need = states + shared * rows;
    if (need && (st = op_pointer("workspace", workspace, 16)) != CCQ_OK) return st;
    if (workspace_bytes < need)
        return op_fail(CCQ_ERR_INVALID_ARG, "workspace of %zu bytes, needs %zu", workspace_bytes, need);
    for (int i = 0; i < 3 && B * T; ++i)
        if (out[i]->p == out[(i + 1) % 3]->p)
            return op_fail(CCQ_ERR_INVALID_ARG, "%s is %s", outs[(i + 1) % 3], outs[i]);
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j)
            if ((st = check_apart(outs[i], *out[i], names[j], *in[j], dtype_bytes(dtype), B, T, d)) != CCQ_OK) return st;
        if ((st = check_apart(outs[(i + 1) % 3], *out[(i + 1) % 3], outs[i], *out[i], dtype_bytes(dtype), B, T, d)) != CCQ_OK) return st;
    }
    const size_t state_bytes = static_cast<size_t>(num_seqs) * H * d * d * 4;
    if ((st = check_states_apart("S0", S0, "dS0", dS0, state_bytes, false)) != CCQ_OK) return st;
    if ((st = check_states_apart("dST", dST, "dS0", dS0, state_bytes, false)) != CCQ_OK) return st;
    if (num_seqs == 0 && !(cu && T)) return CCQ_OK;
    if ((st = op_status_word(&a.status)) != CCQ_OK) return st;
    a.passes = 3;
    const DecayView Q = view_of(*q, H), K = view_of(*k, H), V = view_of(*v, H), O = view_of(*dout, H);
    a.pass[0].q = O;
    a.pass[0].k = V;
    a.pass[0].v = K;
    a.pass[1].q = V;
    a.pass[1].k = O;
    a.pass[1].v = Q;
    a.pass[2].q = K;
    a.pass[2].k = Q;
    a.pass[2].v = O;
    uint8_t *part = static_cast<uint8_t *>(workspace) + states;
    SumArgs sum = {};
    for (int i = 0; i < 3; ++i) {
        DecayPass &p = a.pass[i];
        p.p_scale = scale;
        p.k_scale = i ? scale : 1.f;
        p.s_scale = i ? 1.f : scale;
        p.descending = i > 0;
        p.state_in = i ? dST : S0;
        p.state_out = i == 2 ? dS0 : nullptr;
        p.transposed = i < 2;
        p.kind = i > 0;
        p.parts_transposed = i == 1;
        if (out[i]->heads < H) {
            p.o = part;
            p.o_fp32 = 1;
            p.o_head = d;
            p.o_token = static_cast<int64_t>(H) * d;
            p.o_batch = p.o_token * T;
            const int n = sum.count++;
            sum.parts[n] = reinterpret_cast<const float *>(part);
            sum.out[n] = out[i]->p;
            sum.batch[n] = out[i]->batch;
            sum.token[n] = out[i]->token;
            sum.head[n] = out[i]->head;
            sum.share[n] = static_cast<int>(H / out[i]->heads);
            part += rows;
        } else {
            p.o = out[i]->p;
            p.o_batch = out[i]->batch;
            p.o_token = out[i]->token;
            p.o_head = out[i]->head;
        }
    }
    a.H = H;
    a.d = d;
    a.T = T;
    a.sequences = static_cast<int>(num_seqs);
    a.log_decay = log_decay;
    a.cu = cu;
    a.cu_bytes = cu_bytes;
    a.parts = static_cast<float *>(workspace);
    a.vec = access == 16 && access_out == 16;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // Tokens of no sequence have no gradient: zeros where the passes write (the parts of shared heads, which are summed over all
    // rows, among them).
    if (cu && T) {
        OutsideArgs rest = {};
        for (int i = 0; i < 3; ++i) {
            const DecayPass &p = a.pass[i];
            rest.x[rest.count++] = outside_tensor(p.o, p.o_fp32 ? 4 : dtype_bytes(dtype), p.o_token, p.o_head, H, d);
        }
        rest.T = T;
        rest.cu = cu;
        rest.cu_bytes = cu_bytes;
        rest.sequences = num_seqs;
        if ((st = op_cuda(launch_outside(rest, s), "rows outside launch")) != CCQ_OK) return st;
    }
    bool cores = dtype == CCQ_BF16 && a.vec && B * T > 0;
    for (int i = 0; i < 4; ++i) cores = cores && steps(*in[i], B, T) && (i > 2 || steps(*out[i], B, T));
    if (num_seqs && (st = run_passes(a, plan, dtype, cores, B, 5u, s)) != CCQ_OK) return st;
    if (!sum.count || !(B * T)) return CCQ_OK;
    sum.H = H;
    sum.d = d;
    sum.rows = B * T;
    sum.T = T;
    const unsigned grid = sum.count * static_cast<unsigned>(std::min<int64_t>((sum.rows * H * d / 4 + 255) / 256, 16 * sm_count_now()));
    return op_cuda(dtype == CCQ_BF16 ? launch_after(decay_sum_kernel<__nv_bfloat16>, grid, 256, 0, s, sum, access_out == 16)
                                     : launch_after(decay_sum_kernel<float>, grid, 256, 0, s, sum, access_out == 16),
                   "shared heads' sum launch");
}

}  // extern "C"

// ccq_decay.cuh -- what the kernels of linear attention with a decay for each head share (ccq_ops.h).
//
// One pass over the tokens of a sequence, in ascending or descending order, serves the forward and all of the backward.
// With factors g^n, a pass over (q, k, v) gives
//   o_i = p_scale sum over j up to i of g^|i - j| (q_i . k_j) v_j + s_scale g^(..) S^T q_i,
// S being the state that the tokens before the block have left, and
//   forward   (q, k, v) ascending                 -> o,  S_T
//   dq        (dout, v, k) ascending, S transposed -> dq
//   dk        (v, dout, q) descending, dS transposed -> dk
//   dv        (k, q, dout) descending              -> dv, dS_0
// Descending, S is g times the gradient of the state after the token to the right (dS_T at the last), so that a block of n
// tokens, m tokens passed, reads it with g^m where the ascending pass has g^(m + 1), and adds a token to it with
// k_scale g^(n - m) where that one has g^(n - 1 - m).
#pragma once

#include "ccq_ops.cuh"

namespace ccq {

struct DecayView {
    const void *p;
    int64_t batch, token, head;
    int share;  // heads of the call that read a head of this one
    bool operator==(const DecayView &x) const {
        return p == x.p && batch == x.batch && token == x.token && head == x.head && share == x.share;
    }
};

struct DecayPass {
    DecayView q, k, v;
    void *o;
    int64_t o_batch, o_token, o_head;
    int o_fp32;           // partial gradients of shared heads: fp32 in the workspace
    const float *state_in;  // [sequences][H][d][d] or NULL
    float *state_out;       // or NULL
    int transposed;         // state_in, and the parts of segments, are read transposed
    int descending;
    float p_scale, k_scale, s_scale;
    int kind, parts_transposed;  // whose segments' states it starts from, and how it reads them
};

struct DecayArgs {
    DecayPass pass[3];
    int passes;
    int H, d;
    int64_t T;          // of a sequence, or of all packed ones
    int sequences;
    const float *log_decay;
    const void *cu;
    int cu_bytes;
    int *status;
    // Segments of a sequence, in the order of a pass.  With more than one, a launch with parts_only = 1 leaves in
    // parts[kind][sequence][H][segments][d][d] first the pass's state_in, then what each segment but the last adds to a
    // state from zero, and the segments of the second launch start from these (state_out may be state_in for that reason).
    // Passes from split_pass on of the last split_pairs (sequence, head) pairs run in segments, everything else whole; parts are
    // those of these pairs.
    int segments;
    int split_pairs, split_pass;
    float *parts;
    int parts_only;
    int exact_state;    // a pass hands its states out
    int vec;            // every address and stride is a multiple of 16 bytes
};

// The tokens of a sequence: rows begin .. begin + length of batch row b.
struct DecaySpan {
    int64_t b, begin;
    int64_t length;
};

__device__ __forceinline__ DecaySpan decay_span(const DecayArgs &a, int sequence) {
    DecaySpan s;
    if (!a.cu) {
        s.b = sequence;
        s.begin = 0;
        s.length = a.T;
        return s;
    }
    const int64_t from = load_index(a.cu, a.cu_bytes, sequence), to = load_index(a.cu, a.cu_bytes, sequence + 1);
    s.b = 0;
    s.begin = min(max(from, static_cast<int64_t>(0)), a.T);
    const int64_t end = min(max(to, s.begin), a.T);
    s.length = end - s.begin;
    if ((s.begin != from || end != to) && threadIdx.x == 0) note_index(a.status);
    return s;
}

// Packed sequences in the order of their lengths, the longest first, so that no long one is left for the end: the sequence of
// rank `rank` (up to 256 of them, a few hundred operations a thread; more are taken as they lie).  `scratch`: 257 ints of shared
// memory; all threads of the block, two barriers.  64 prompts of 100 to 4000 tokens, 16 heads of 128, the longest last:
// 302 us as they lie, 244 so.
constexpr int kRanked = 256;
__device__ __forceinline__ int decay_longest_first(const DecayArgs &a, int rank, int *scratch) {
    if (!a.cu || a.sequences > kRanked || a.sequences < 2) return rank;
    for (int i = threadIdx.x; i < a.sequences; i += blockDim.x) {
        const int64_t n = load_index(a.cu, a.cu_bytes, i + 1) - load_index(a.cu, a.cu_bytes, i);
        scratch[i] = static_cast<int>(min(max(n, static_cast<int64_t>(0)), static_cast<int64_t>(0x7fffffff)));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.sequences; i += blockDim.x) {
        int longer = 0;
        for (int j = 0; j < a.sequences; ++j) longer += scratch[j] > scratch[i] || (scratch[j] == scratch[i] && j < i);
        if (longer == rank) scratch[kRanked] = i;
    }
    __syncthreads();
    return scratch[kRanked];
}

// The logarithm of a head's decay g, and log2 g as two floats.  A decay below 2^-199 keeps nothing in fp32 either way (and
// -inf would give NaN as g^0).
struct DecayLog {
    float natural, hi, lo;
};
__device__ __forceinline__ DecayLog decay_log2(const float *log_decay, int h) {
    constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.9259629911266175e-8f;
    DecayLog l;
    l.natural = log_decay[h] < -138.f ? -138.f : log_decay[h];
    l.hi = l.natural * kLog2e;
    l.lo = fmaf(l.natural, kLog2e, -l.hi) + l.natural * kLog2eLow;
    return l;
}

// g^n within 2^-22 of itself: the exponent's rounding is put back as a factor.
__device__ __forceinline__ float decay_power(const DecayLog &l, int n) {
    const float x = l.hi * n, rest = fmaf(l.hi, static_cast<float>(n), -x) + l.lo * n;
    const float p = exp2f(x);
    return fmaf(p, rest * 0.6931471805599453f, p);
}

// g^n as two floats: the factor of the state at every block, whose error would add up over a sequence.
__device__ __forceinline__ float2 decay_keep(const DecayLog &l, int n) {
    const double p = exp(static_cast<double>(l.natural) * n);
    const float hi = static_cast<float>(p);
    return make_float2(hi, static_cast<float>(p - hi));
}

// g as two floats, within 2^-23 log(g)^2 + 2^-49 of itself, without 64-bit arithmetic for slow decays (whose error would add up over the most
// tokens): 1 + x + x^2 (1/2 + x/6 + ..), x exact, by the series of exp.
__device__ __forceinline__ float2 decay_factor(const DecayLog &l) {
    const float x = l.natural;
    if (!(x >= -0.25f && x <= 0.f)) return decay_keep(l, 1);
    float q = 1.f / 40320.f;
    q = fmaf(q, x, 1.f / 5040.f);
    q = fmaf(q, x, 1.f / 720.f);
    q = fmaf(q, x, 1.f / 120.f);
    q = fmaf(q, x, 1.f / 24.f);
    q = fmaf(q, x, 1.f / 6.f);
    q = fmaf(q, x, 0.5f);
    q *= x * x;
    const float first = 1.f + x, rest = (x - (first - 1.f)) + q, hi = first + rest;
    return make_float2(hi, rest - (hi - first));
}

// Lets the launch after this one start where SMs are free.
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Where the state of (sequence, head, segment) lies among the parts.
__device__ __forceinline__ int64_t decay_part(const DecayArgs &a, int kind, int sequence, int h, int segment) {
    const int64_t pair = static_cast<int64_t>(sequence) * a.H + h - (static_cast<int64_t>(a.sequences) * a.H - a.split_pairs);
    return ((static_cast<int64_t>(kind) * a.split_pairs + pair) * a.segments + segment) * a.d * a.d;
}

// Tensors of [T, heads, width], strides in bytes, whose rows outside all packed sequences become zeros.
struct OutsideTensor {
    void *p;
    int64_t token, head;
    int heads, bytes;  // of a head's row
    int wide;          // in accesses of 16 bytes
};
struct OutsideArgs {
    OutsideTensor x[3];
    int count;
    int64_t T;
    const void *cu;
    int cu_bytes;
    int64_t sequences;
};
OutsideTensor outside_tensor(void *p, int elem, int64_t token, int64_t head, int heads, int width);  // (strides in elements)
cudaError_t launch_outside(const OutsideArgs &a, cudaStream_t s);

cudaError_t launch_decay_chunks(const DecayArgs &a, int64_t B, cudaStream_t s);  // bf16 on the tensor cores
cudaError_t launch_decay_blocks(const DecayArgs &a, ccq_dtype dtype, cudaStream_t s);

}  // namespace ccq

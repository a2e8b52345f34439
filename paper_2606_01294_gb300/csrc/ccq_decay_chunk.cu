// ccq_decay_chunk.cu -- linear attention with a decay for each head on the tensor cores (bf16; ccq_decay.cuh says how one pass
// serves the forward and the gradients).
//
// A CTA walks the chunks of 128 tokens of one (pass, sequence, head, segment).  With g^n the powers of the head's decay:
//   A  = Q K^T                 tcgen05, 128 x 128 x d
//   P  = A . p_scale g^|i - j| on the kept side of the diagonal, rounded to bf16, in tensor memory (an A operand there)
//   O1 = Q S                   128 x d x d, S the state before the chunk rounded to bf16
//   O2 = P V                   128 x d x 128
//   o_i = s_scale g^(i + 1) O1_i + O2_i            (descending: g^(n - 1 - i))
//   D  = W^T V                 d x d x 128 three times: W = diag(k_scale g^(n - 1 - j)) K in three bf16 terms, all its 24 bits
//   S  = g^n S + D             in registers, fp32
// Nothing of this is a chain through the chunk but S itself, and D of a chunk does not depend on S: products, the two
// kinds of epilogue warps and the loads work on neighbouring chunks at the same time.
//   ATT   (warps 0-7)   P from A, o from O1 and O2 (thread: a row, half of its columns)
//   STATE (warps 8-15)  W from K, S from D, and S's bf16 copy for the next chunk
//   ISSUE (warp 16)     one thread issues the products in the order QK, QS, W^T V, PV
//   LOAD  (warp 17)     one thread issues the TMA loads; a tile is loaded again when its last product has read it
// Rows past a sequence's end: TMA gives zeros past the tensor; rows of other packed sequences get W = 0, P = 0, and
// zeros in V (0 times what is not finite would not be 0).
#include <string.h>

#include "ccq_decay.cuh"

namespace ccq {
namespace {

constexpr int kC = 128;  // tokens of a chunk
constexpr int kAttWarps = 8, kStateWarps = 8;
constexpr int kStateWarp0 = kAttWarps, kIssueWarp = kAttWarps + kStateWarps, kLoadWarp = kIssueWarp + 1;
constexpr int kThreads = 32 * (kLoadWarp + 1);  // 576
constexpr int kBlockBytes = kC * 128;           // a T64 tile of 128 tokens

template <int D> struct Map {
    static constexpr uint32_t kTile = kBlockBytes * (D / 64);  // [128 tokens][D]
    static constexpr uint32_t kQ = 0, kK = kTile, kV = 2 * kTile, kW = 3 * kTile;  // W: three tiles
    static constexpr uint32_t kS = 6 * kTile;                  // [D][D]
    static constexpr uint32_t kTable = kS + D * D * 2;         // [256] p_scale g^(e - 127), 0 for e < 127
    static constexpr uint32_t kBars = kTable + 1024;
    static constexpr uint32_t kMisc = kBars + 16 * 8;          // tmem address, abort flag, keep[2] as two floats each
    static constexpr uint32_t kBytes = kMisc + 32 + 1024;      // and the alignment's slack
};
static_assert(Map<128>::kBytes <= 232448, "exceeds the 227 KB of a CTA");

enum { BAR_Q, BAR_K, BAR_V, BAR_A, BAR_O1, BAR_D, BAR_O2, BAR_P, BAR_OFREE, BAR_W, BAR_S, kBars };
static_assert(kBars <= 16, "barrier area");

constexpr uint32_t TM_A = 0, TM_O1 = 128, TM_O2 = 256, TM_D = 384, kTmemCols = 512;

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

// D[tmem] (+)= A[tmem] * B[smem], bf16 operands: A's row is its lane, two elements of K a column.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

struct ChunkMapsOf {
    CUtensorMap q, k, v;
};
struct DecayMaps {
    ChunkMapsOf pass[3];
};

// w in three bf16 terms of two elements each.
__device__ __forceinline__ void split3(float a, float b, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
    hi = pack_bf16(a, b);
    const float ra = a - __uint_as_float(hi << 16), rb = b - __uint_as_float(hi & 0xffff0000u);
    mid = pack_bf16(ra, rb);
    lo = pack_bf16(ra - __uint_as_float(mid << 16), rb - __uint_as_float(mid & 0xffff0000u));
}

template <int D, bool PARTS>
__global__ void __maxnreg__(96) decay_chunk_kernel(const __grid_constant__ DecayMaps maps, const __grid_constant__ DecayArgs a) {
    using M = Map<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = smem_align1024(smem_raw);
    const uint32_t sb = smem_addr(sm);
    float *table = reinterpret_cast<float *>(sm + M::kTable);
    uint64_t *bar = reinterpret_cast<uint64_t *>(sm + M::kBars);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(sm + M::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(sm + M::kMisc + 4);
    float2 *keeps = reinterpret_cast<float2 *>(sm + M::kMisc + 8);  // g^128 and g^n of the ragged chunk, as two floats

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    unsigned x = blockIdx.x;
    const int pi = x % a.passes;
    x /= a.passes;
    const int nseg = PARTS ? a.segments - 1 : a.segments;
    const int segment = x % nseg;
    x /= nseg;
    const int h = x % a.H, sequence = x / a.H;
    const DecayPass &ps = a.pass[pi];
    const ChunkMapsOf &mp = maps.pass[pi];
    const bool down = ps.descending != 0;
    const DecaySpan span = decay_span(a, sequence);
    const int length = static_cast<int>(span.length);
    const int chunks = (length + kC - 1) / kC, per = (chunks + a.segments - 1) / a.segments;
    const int first = min(per * segment, chunks), count = min(first + per, chunks) - first;
    const int ragged = length - (chunks - 1) * kC;  // tokens of the sequence's last chunk
    const DecayLog l2 = decay_log2(a.log_decay, h);
    // chunk r of the segment: its first token within the sequence, its tokens
    auto chunk_at = [&](int r) { return (down ? chunks - 1 - (first + r) : first + r); };
    auto begin_of = [&](int r) { return chunk_at(r) * kC; };
    auto tokens_of = [&](int r) { return chunk_at(r) == chunks - 1 ? ragged : kC; };
    int *status = a.status;

    if (tid == 0) {
        for (int i = 0; i < kBars; ++i)
            mbar_init(&bar[i], i == BAR_P || i == BAR_OFREE ? kAttWarps : i == BAR_W || i == BAR_S ? kStateWarps : 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0) tmem_alloc(tmem_slot, kTmemCols);
    if (!PARTS && tid < 256) table[tid] = tid < 127 ? 0.f : ps.p_scale * decay_power(l2, tid - 127);
    if (tid >= kThreads - 2) {
        keeps[tid - (kThreads - 2)] = decay_keep(l2, tid == kThreads - 2 ? kC : ragged);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = *tmem_slot;
    const uint32_t tq = tbase + (static_cast<uint32_t>(32 * (warp & 3)) << 16);  // the warp's lane quadrant

    if (warp < kAttWarps) {
        // ============================================================ ATT
        if (!PARTS) {
            const int half = warp >> 2, i = 32 * (warp & 3) + lane;  // row, column half
            const int row0 = 32 * (warp & 3);
            const float near = decay_power(l2, i + 1) * ps.s_scale;  // ascending, or a full chunk's mirror image below
            const float far = decay_power(l2, kC - 1 - i) * ps.s_scale;
            for (int r = 0; r < count; ++r) {
                const uint32_t par = r & 1;
                const int n = tokens_of(r);
                mbar_wait(&bar[BAR_A], par, abort_flag, status);
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int j0 = 64 * half + 32 * c;
                    uint32_t p[16];
                    if (down ? j0 + 31 < row0 || j0 >= n : j0 > row0 + 31) {  // nothing kept
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[e] = 0;
                    } else {
                        float v[32];
                        tmem_ld32(tq + TM_A + j0, v);
                        const float *t = table + 127 + (down ? j0 - i : i - j0);
                        if (down) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                const float f = t[e];
                                v[e] = f != 0.f && j0 + e < n ? v[e] * f : 0.f;
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                const float f = t[-e];
                                v[e] = f != 0.f ? v[e] * f : 0.f;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                    }
                    tmem_st16(tq + TM_A + 64 * half + 16 * c, p);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar[BAR_P]);

                const float fac = down ? (n == kC ? far : i < n ? decay_power(l2, n - 1 - i) * ps.s_scale : 0.f) : near;
                const int64_t at = span.b * ps.o_batch + (span.begin + begin_of(r) + i) * ps.o_token + h * ps.o_head +
                                   half * (D / 2);
                mbar_wait(&bar[BAR_O1], par, abort_flag, status);
                mbar_wait(&bar[BAR_O2], par, abort_flag, status);
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    float u[32], w[32];
                    tmem_ld32(tq + TM_O1 + half * (D / 2) + 32 * c, u);
                    tmem_ld32(tq + TM_O2 + half * (D / 2) + 32 * c, w);
                    if (c == D / 64 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bar[BAR_OFREE]);
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) u[e] = u[e] * fac + w[e];
                    if (i < n) {
                        if (ps.o_fp32) {
                            float *to = static_cast<float *>(ps.o) + at + 32 * c;
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                *reinterpret_cast<float4 *>(to + e) = make_float4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                        } else {
                            __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(ps.o) + at + 32 * c;
#pragma unroll
                            for (int e = 0; e < 32; e += 8)
                                *reinterpret_cast<uint4 *>(to + e) =
                                    make_uint4(pack_bf16(u[e], u[e + 1]), pack_bf16(u[e + 2], u[e + 3]),
                                               pack_bf16(u[e + 4], u[e + 5]), pack_bf16(u[e + 6], u[e + 7]));
                        }
                    }
                }
            }
        }
    } else if (warp < kIssueWarp) {
        // ============================================================ STATE
        // S: row `row`, columns col0 .. col0 + kCols.  (d = 64: an accumulator of 64 rows keeps rows 16 q .. in lanes 32 q ..,
        // which the first four warps read, 32 columns a thread.)
        constexpr int kCols = D == 128 ? 64 : 32;
        const int sw = warp - kStateWarp0, st = tid - 32 * kStateWarp0;
        const bool holds = D == 128 || sw < 4;
        const int row = D == 128 ? 32 * (sw & 3) + lane : 16 * (sw & 3) + (lane & 15);
        const int col0 = D == 128 ? 64 * (sw >> 2) : 32 * (lane >> 4);
        float S[kCols];
        auto add = [&](const float *m, bool transposed, float keep) {
            if (transposed) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const float f = m[(col0 + c) * D + row];
                    S[c] = keep == 0.f ? f : S[c] * keep + f;
                }
            } else {
#pragma unroll
                for (int c = 0; c < kCols; c += 4) {
                    const float4 f = *reinterpret_cast<const float4 *>(m + row * D + col0 + c);
                    S[c] = keep == 0.f ? f.x : S[c] * keep + f.x;
                    S[c + 1] = keep == 0.f ? f.y : S[c + 1] * keep + f.y;
                    S[c + 2] = keep == 0.f ? f.z : S[c + 2] * keep + f.z;
                    S[c + 3] = keep == 0.f ? f.w : S[c + 3] * keep + f.w;
                }
            }
        };
        auto put = [&](float *m) {
            if (!holds) return;
#pragma unroll
            for (int c = 0; c < kCols; c += 4)
                *reinterpret_cast<float4 *>(m + row * D + col0 + c) = make_float4(S[c], S[c + 1], S[c + 2], S[c + 3]);
        };
        auto snapshot = [&]() {  // S rounded to bf16, for the next chunk's Q S
            if (holds) {
#pragma unroll
                for (int c = 0; c < kCols; c += 8) {
                    const int col = col0 + c;
                    *reinterpret_cast<uint4 *>(sm + M::kS + (col >> 6) * (D * 128) + t64_chunk(row, (col & 63) >> 3)) =
                        make_uint4(pack_bf16(S[c], S[c + 1]), pack_bf16(S[c + 2], S[c + 3]), pack_bf16(S[c + 4], S[c + 5]),
                                   pack_bf16(S[c + 6], S[c + 7]));
                }
            }
            fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar[BAR_S]);
        };
        auto clear = [&]() {
#pragma unroll
            for (int c = 0; c < kCols; ++c) S[c] = 0.f;
        };
        clear();
        const int64_t matrix = (static_cast<int64_t>(sequence) * a.H + h) * D * D;
        if (a.segments == 1 || (PARTS && segment == 0)) {
            if (ps.state_in) add(ps.state_in + matrix, ps.transposed, 0.f);
            if (PARTS) {
                put(a.parts + decay_part(a, ps.kind, sequence, h, 0));
                clear();
            }
        } else if (!PARTS) {
            for (int g = 0; g <= segment; ++g) {
                const int lo = min(per * (g - 1), chunks), hi = min(per * g, chunks);  // segment g - 1
                int n = 0;
                if (g > 0 && hi > lo) n = (hi - lo) * kC - ((down ? lo == 0 : hi == chunks) ? kC - ragged : 0);
                add(a.parts + decay_part(a, ps.kind, sequence, h, g), ps.parts_transposed,
                    g == 0 ? 0.f : decay_power(l2, n));
            }
        }
        if (!PARTS) snapshot();
        // W: this thread's 16-byte chunk of rows wr + kRows k
        constexpr int kWide = D / 8, kRows = 32 * kStateWarps / kWide;
        const int wc = st % kWide, wr = st / kWide;
        const uint32_t wtile = (wc >> 3) * kBlockBytes;
        for (int r = 0; r < count; ++r) {
            const uint32_t par = r & 1;
            const int n = tokens_of(r);
            mbar_wait(&bar[BAR_K], par, abort_flag, status);
#pragma unroll 2
            for (int k = 0; k < kC / kRows; ++k) {
                const int t = wr + kRows * k;
                const uint32_t off = wtile + t64_chunk(t, wc & 7);
                const uint4 u = *reinterpret_cast<const uint4 *>(sm + M::kK + off);
                float f[8];
                unpack_bf16x8(u, f);
                const float w = decay_power(l2, down ? t + 1 : n - 1 - t) * ps.k_scale;
                uint4 hi = make_uint4(0, 0, 0, 0), mid = hi, lo = hi;
                if (t < n) {
                    split3(f[0] * w, f[1] * w, hi.x, mid.x, lo.x);
                    split3(f[2] * w, f[3] * w, hi.y, mid.y, lo.y);
                    split3(f[4] * w, f[5] * w, hi.z, mid.z, lo.z);
                    split3(f[6] * w, f[7] * w, hi.w, mid.w, lo.w);
                }
                *reinterpret_cast<uint4 *>(sm + M::kW + off) = hi;
                *reinterpret_cast<uint4 *>(sm + M::kW + M::kTile + off) = mid;
                *reinterpret_cast<uint4 *>(sm + M::kW + 2 * M::kTile + off) = lo;
            }
            if (n < kC && a.cu) {  // rows of other sequences
                mbar_wait(&bar[BAR_V], par, abort_flag, status);
                for (int t = n + wr; t < kC; t += kRows)
                    *reinterpret_cast<uint4 *>(sm + M::kV + wtile + t64_chunk(t, wc & 7)) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar[BAR_W]);

            mbar_wait(&bar[BAR_D], par, abort_flag, status);
            tc_fence_after();
            const float2 keep = keeps[chunk_at(r) == chunks - 1];
            if (holds) {
                auto step = [&](float &s, float d) { s = fmaf(s, keep.x, fmaf(s, keep.y, d)); };
                if constexpr (D == 128) {
#pragma unroll
                    for (int c = 0; c < kCols; c += 16) {
                        float d[16];
                        tmem_ld16(tq + TM_D + col0 + c, d);
#pragma unroll
                        for (int e = 0; e < 16; ++e) step(S[c + e], d[e]);
                    }
                } else {
                    float d[32];
                    tmem_ld16x2_32<32>(tq + TM_D, d);
#pragma unroll
                    for (int e = 0; e < 32; ++e) step(S[e], d[e]);
                }
            }
            if (PARTS || r + 1 == count) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar[BAR_S]);
            } else {
                // (Q S of this chunk has read the copy: W^T V, whose end was waited for, was issued after it -- and it is
                // waited for by itself)
                mbar_wait(&bar[BAR_O1], par, abort_flag, status);
                snapshot();
            }
        }
        if (PARTS)
            put(a.parts + decay_part(a, ps.kind, sequence, h, segment + 1));
        else if (ps.state_out && segment == a.segments - 1)
            put(ps.state_out + matrix);
    } else if (warp == kIssueWarp) {
        // ============================================================ ISSUE
        if (lane == 0) {
            constexpr uint32_t kQK = make_idesc(kC, kC, 0, 0), kQS = make_idesc(kC, D, 0, 1), kWV = make_idesc(D, D, 1, 1),
                               kPV = make_idesc(kC, D, 0, 1);
            for (int r = 0; r < count; ++r) {
                const uint32_t par = r & 1, before = par ^ 1;
                if (!PARTS) {
                    mbar_wait(&bar[BAR_Q], par, abort_flag, status);
                    mbar_wait(&bar[BAR_K], par, abort_flag, status);
                    if (r) mbar_wait(&bar[BAR_O2], before, abort_flag, status);  // P V has read P, which lies in A
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_bf16(tbase + TM_A, desc_kmajor(sb + M::kQ + (k >> 2) * kBlockBytes, k & 3),
                                 desc_kmajor(sb + M::kK + (k >> 2) * kBlockBytes, k & 3), kQK, k > 0);
                    mma_commit(&bar[BAR_A]);
                    mbar_wait(&bar[BAR_S], par, abort_flag, status);
                    if (r) mbar_wait(&bar[BAR_OFREE], before, abort_flag, status);
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_bf16(tbase + TM_O1, desc_kmajor(sb + M::kQ + (k >> 2) * kBlockBytes, k & 3),
                                 desc_mnmajor(sb + M::kS, D * 128, k), kQS, k > 0);
                    mma_commit(&bar[BAR_O1]);
                } else if (r) {
                    mbar_wait(&bar[BAR_S], before, abort_flag, status);  // D has been read
                }
                mbar_wait(&bar[BAR_V], par, abort_flag, status);
                mbar_wait(&bar[BAR_W], par, abort_flag, status);
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < kC / 16; ++k)
#pragma unroll
                    for (int t = 2; t >= 0; --t)  // the small terms first
                        mma_bf16(tbase + TM_D, desc_mnmajor(sb + M::kW + t * M::kTile, kBlockBytes, k),
                                 desc_mnmajor(sb + M::kV, kBlockBytes, k), kWV, k > 0 || t < 2);
                mma_commit(&bar[BAR_D]);
                if (!PARTS) {
                    mbar_wait(&bar[BAR_P], par, abort_flag, status);
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < kC / 16; ++k)
                        mma_bf16_ts(tbase + TM_O2, tbase + TM_A + 64 * (k >> 2) + 8 * (k & 3),
                                    desc_mnmajor(sb + M::kV, kBlockBytes, k), kPV, k > 0);
                    mma_commit(&bar[BAR_O2]);
                }
            }
        }
    } else {
        // ============================================================ LOAD
        if (lane == 0) {
            const int hq = h / ps.q.share, hk = h / ps.k.share, hv = h / ps.v.share, b = static_cast<int>(span.b);
            auto load = [&](const CUtensorMap *map, uint32_t to, int which, int head, int token) {
                mbar_arrive_expect_tx(&bar[which], M::kTile);
#pragma unroll
                for (int c = 0; c < D / 64; ++c)
                    tma_load_4d(sm + to + c * kBlockBytes, map, &bar[which], 64 * c, head, token, b);
            };
            auto prefetch = [&](const CUtensorMap *map, int head, int token) {
#pragma unroll
                for (int c = 0; c < D / 64; ++c) tma_prefetch_l2_4d(map, 64 * c, head, token, b);
            };
            tma_prefetch_desc(&mp.k);
            tma_prefetch_desc(&mp.v);
            if (!PARTS) tma_prefetch_desc(&mp.q);
            for (int r = 0; r < count; ++r) {
                const uint32_t before = (r & 1) ^ 1;
                const int token = static_cast<int>(span.begin) + begin_of(r);
                if (r) {
                    mbar_wait(&bar[BAR_W], before, abort_flag, status);
                    if (!PARTS) mbar_wait(&bar[BAR_A], before, abort_flag, status);
                }
                load(&mp.k, M::kK, BAR_K, hk, token);
                if (!PARTS) {
                    if (r) mbar_wait(&bar[BAR_O1], before, abort_flag, status);
                    load(&mp.q, M::kQ, BAR_Q, hq, token);
                }
                if (r + 1 < count) {  // the next chunk into L2, so that its loads are short
                    const int next = static_cast<int>(span.begin) + begin_of(r + 1);
                    prefetch(&mp.k, hk, next);
                    if (!PARTS) prefetch(&mp.q, hq, next);
                    prefetch(&mp.v, hv, next);
                }
                if (r) {
                    mbar_wait(&bar[BAR_D], before, abort_flag, status);
                    if (!PARTS) mbar_wait(&bar[BAR_O2], before, abort_flag, status);
                }
                load(&mp.v, M::kV, BAR_V, hv, token);
            }
            // no CTA leaves before its copies have landed (after a wait that ran out)
            if (count > 0) {
                const uint32_t last = (count - 1) & 1;
                mbar_drain(&bar[BAR_K], last);
                mbar_drain(&bar[BAR_V], last);
                if (!PARTS) mbar_drain(&bar[BAR_Q], last);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tbase, kTmemCols);
}

template <int D, bool PARTS> cudaError_t launch(const DecayMaps &m, const DecayArgs &a, cudaStream_t s) {
    constexpr int kBytes = Map<D>::kBytes;
    cudaError_t e = allow_shared<decay_chunk_kernel<D, PARTS>>(kBytes);
    if (e != cudaSuccess) return e;
    const int64_t grid = static_cast<int64_t>(PARTS ? a.segments - 1 : a.segments) * a.H * a.sequences * a.passes;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    decay_chunk_kernel<D, PARTS><<<static_cast<unsigned>(grid), kThreads, kBytes, s>>>(m, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_decay_chunks(const DecayArgs &a, int64_t B, cudaStream_t s) {
    DecayMaps m;
    const DecayView *seen[9];
    const CUtensorMap *made[9];
    int count = 0;
    for (int i = 0; i < a.passes; ++i) {
        const DecayView *views[3] = {&a.pass[i].q, &a.pass[i].k, &a.pass[i].v};
        CUtensorMap *to[3] = {&m.pass[i].q, &m.pass[i].k, &m.pass[i].v};
        for (int j = 0; j < 3; ++j) {
            const DecayView &x = *views[j];
            int k = 0;  // (the gradients' passes read the same tensors)
            while (k < count && memcmp(seen[k], &x, sizeof x)) ++k;
            if (k < count) {
                *to[j] = *made[k];
                continue;
            }
            if (!make_heads_map(to[j], x.p, B, a.T, a.H / x.share, a.d, x.batch, x.token, x.head, kC))
                return cudaErrorInvalidValue;
            seen[count] = &x;
            made[count++] = to[j];
        }
    }
    if (a.parts_only) return a.d == 128 ? launch<128, true>(m, a, s) : launch<64, true>(m, a, s);
    return a.d == 128 ? launch<128, false>(m, a, s) : launch<64, false>(m, a, s);
}

}  // namespace ccq

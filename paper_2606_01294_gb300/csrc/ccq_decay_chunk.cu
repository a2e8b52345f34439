// ccq_decay_chunk.cu -- linear attention with a decay for each head on the tensor cores (bf16; ccq_decay.cuh says how one pass
// serves the forward and the gradients).
//
// A CTA walks the chunks of 128 tokens of one (pass, sequence, head, segment).  With g^n the powers of the head's decay:
//   A  = Q K^T                 tcgen05, 128 x 128 x d
//   P  = A . p_scale g^|i - j| on the kept side of the diagonal, rounded to bf16, in tensor memory (an A operand there)
//   O1 = Q S                   128 x d x d, S the state before the chunk rounded to bf16
//   O2 = P V                   128 x d x 128
//   o_i = s_scale g^(i + 1) O1_i + O2_i            (descending: g^(n - 1 - i))
//   D  = V^T W                 d x d x 128 three times: W = diag(k_scale g^(n - 1 - j)) K in three bf16 terms, all its 24 bits
//   S^T = g^n S^T + D          in registers, fp32
// Nothing of this is a chain through the chunk but S itself, and D of a chunk does not depend on S: products, the two
// kinds of epilogue warps and the loads work on neighbouring chunks at the same time.
//   SP    (warps 0-7)   S from D and its bf16 copy, then P from A (thread: a row, half of its columns)
//   W     (warps 8-15)  W from K, 32 tokens at a time in two slots
//   O     (warps 16-19) o from O1 and O2 (thread: a row), stored by TMA from a tile
//   ISSUE (warps 20, 22) one thread issues QK, QS and PV, another V^T W: a thread waits while its products run, so that with one
//                       alone the tensor cores would stand still between them
//   LOAD  (warp 21)     one thread issues the TMA loads: a tile is loaded again when its last reader is through with it;
//                       V in halves of 64 tokens, K in a ring of three halves
// Bound by the steps of a chunk one after another, 3.4 us at d = 128 and 2.4 at 64, D through registers to S and its copy and A to P
// among them, not by a unit: HBM 74 % of a copy, the tensor cores 40 to 53 %, issue 50 %; W, the longest stage, is 12 %.  bf16, 16 heads of 128: 8 x 4096 tokens 109 us
// (decay_block_kernel: 3150), 1 x 20480 in segments 122, 64 packed prompts 241, gradients of 4 x 4096 172.  Why so: chunks of
// 128 fill an accumulator's lanes; S stays in registers, as in tensor memory it would be read, scaled and written there each
// chunk; a head has one CTA, for with two halves of V's columns both would form P and the split.
// What is rounded to fewer bits than fp32: P and the copy of S that queries read, as bf16 operands (relative error of o against 64 bits 2.3e-3;
// 1.7e-3 where o alone is rounded).  In two bf16 terms each they would cost P V and Q S twice, a third more products, and S's second term 32 KB
// of shared memory, of which none is left at d = 128.  S itself is not rounded: fp32, its factors two floats, its increment's terms as below.
// Rows past a sequence's end: TMA gives zeros past the tensor; rows of other packed sequences get W = 0, P = 0, and
// zeros in V (0 times what is not finite would not be 0).
#include "ccq_decay.cuh"

namespace ccq {
namespace {

constexpr int kC = 128;  // tokens of a chunk
constexpr int kAhead = 1;  // chunks
constexpr int kWarps = 8;  // SP's and W's
constexpr int kOWarps = 4;
constexpr int kWWarp0 = kWarps, kOWarp0 = 2 * kWarps, kIssueWarp = kOWarp0 + kOWarps, kLoadWarp = kIssueWarp + 1,
              kIssueWWarp = kIssueWarp + 2, kKeepWarp = kIssueWarp + 3;
constexpr int kThreads = 32 * 24;  // six warpgroups
// Registers a thread: 80 at launch, then as the warps' work wants them, 480 for the six warpgroups together.
constexpr int kSpRegs = 120, kWRegs = 56, kORegs = 72, kOtherRegs = 56;
constexpr int kLaunchRegs = 80;
static_assert(2 * kSpRegs + 2 * kWRegs + kORegs + kOtherRegs <= 6 * kLaunchRegs, "more registers than the launch has");
static_assert(kSpRegs >= kLaunchRegs && kWRegs <= kLaunchRegs && kORegs <= kLaunchRegs && kOtherRegs <= kLaunchRegs,
              "one kind of warps takes registers, the others give them");

enum { kOutBar = 1, kKeepBar = 2 };  // named barriers

template <int D> struct Map {
    static constexpr uint32_t kBlocks = D / 64;                 // T64 tiles side by side
    static constexpr uint32_t kBlock = kC * 128;                // of 128 tokens
    static constexpr uint32_t kTile = kBlock * kBlocks;         // [128 tokens][D]
    static constexpr uint32_t kHBlock = 64 * 128, kHalf = kHBlock * kBlocks;  // of 64 tokens
    static constexpr uint32_t kWBlock = 32 * 128, kWTerm = kWBlock * kBlocks, kWSlot = 3 * kWTerm;
    static constexpr uint32_t kQ = 0, kO = kTile;               // o: two blocks, of 64 columns in bf16, 32 in fp32
    static constexpr uint32_t kV = kO + 2 * kBlock;             // two halves
    static constexpr uint32_t kK = kV + kTile;                  // three halves, [d / 64][half][64 tokens]
    static constexpr uint32_t kKBlock = 3 * kHBlock;
    static constexpr uint32_t kW = kK + 3 * kHalf;              // two slots of 32 tokens, three terms each
    static constexpr uint32_t kS = kW + 2 * kWSlot;             // [D][D]
    static constexpr uint32_t kTable = kS + D * D * 2;          // [256] p_scale g^(e - 127), 0 for e < 127
    static constexpr uint32_t kPowers = kTable + 1024;          // [129] k_scale g^e
    static constexpr uint32_t kColumn = kPowers + 528;          // [32] g^(31 - e), descending g^e
    static constexpr uint32_t kBars = kColumn + 128;
    static constexpr uint32_t kMisc = kBars + 24 * 8;           // tmem address, abort flag, keep[2] as two floats each
    static constexpr uint32_t kBytes = kMisc + 32 + 1024;       // and the alignment's slack
};
static_assert(Map<128>::kBytes <= 232448, "exceeds the 227 KB of a CTA");

enum {
    BAR_Q, BAR_K, BAR_V = BAR_K + 3, BAR_KFREE = BAR_V + 2, BAR_VFREE = BAR_KFREE + 3, BAR_W = BAR_VFREE + 2,
    BAR_WFREE = BAR_W + 2, BAR_A = BAR_WFREE + 2, BAR_O1, BAR_D, BAR_O2, BAR_P, BAR_OFREE, BAR_S, BAR_DFREE, BAR_ZEROS, kBars
};
static_assert(kBars <= 24, "barrier area");

constexpr uint32_t TM_A = 0, TM_O1 = 128, TM_O2 = 256, TM_D = 384, kTmemCols = 512;

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

// mbar_wait whose first try is all that a wait on a phase that is complete costs.
__device__ __forceinline__ void wait_for(uint64_t *bar, uint32_t parity, volatile int *abort, int *status) {
    const uint32_t at = smem_addr(bar);
    if (mbar_try_wait(at, parity)) return;
    const long long start = clock64();
    while (!mbar_try_wait(at, parity)) {
        if (*abort) return;
        if (clock64() - start > kWaitLimitCycles) {
            *abort = 1;
            atomicExch(status, kStatusTimeout);
            return;
        }
    }
}

// 16 columns of two places, waited for together: a round trip to tensor memory beside the products takes a few hundred cycles.
__device__ __forceinline__ void tmem_ld16_two(uint32_t at0, uint32_t at1, float (&u)[16], float (&w)[16]) {
    uint32_t r[16], q[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(q[0]), "=r"(q[1]),
          "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7]), "=r"(q[8]), "=r"(q[9]), "=r"(q[10]),
          "=r"(q[11]), "=r"(q[12]), "=r"(q[13]), "=r"(q[14]), "=r"(q[15])
        : "r"(at0), "r"(at1)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        u[i] = __uint_as_float(r[i]);
        w[i] = __uint_as_float(q[i]);
    }
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

template <int N> __device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N> __device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// One thread of a warp that runs together.  (The compiler then knows of one thread and keeps what it issues in uniform registers:
// gradients of 3 x 4096 tokens, 16 heads of 64 90 us with `lane == 0`, 79 so.)
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p;
}

// The place of the next half of K in its ring of three.
struct Ring {
    int slot = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() {
        slot = slot == 2 ? 0 : slot + 1;
        parity ^= slot == 0;
    }
};

struct ChunkMapsOf {
    CUtensorMap q, k, v, o;
};
struct DecayMaps {
    ChunkMapsOf pass[3];
};

// Two values in three bf16 terms each, the bits of 24 from the top: cutting off leaves differences that are exact.
// In two terms they are rounded, the second within 2^-17 of the value.
template <int TERMS> __device__ __forceinline__ void split(uint64_t x, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
    const uint64_t minus = f2_make(-1.f, -1.f);
    auto top = [](uint64_t v) { return __byte_perm(static_cast<uint32_t>(v), static_cast<uint32_t>(v >> 32), 0x7632); };
    hi = TERMS == 2 ? bf16x2_from_f2(x) : top(x);
    x = f2_fma(f2_from_bf16x2(hi), minus, x);
    mid = TERMS == 2 ? bf16x2_from_f2(x) : top(x);
    if (TERMS == 3) lo = top(f2_fma(f2_from_bf16x2(mid), minus, x));
}

// TERMS: of W.  Three where a state is handed out (its error then is that of fp32 sums), two where the state serves the outputs
// alone, which read it rounded to bf16: gradients of 4 x 4096 x 16 x 128 214 us with three, 199 with two.
// SUMS: some passes leave parts of shared heads' gradients, in fp32 (without their code the others run 4 % faster).
template <int D, bool PARTS, int TERMS, bool SUMS>
__global__ void __maxnreg__(kLaunchRegs) decay_chunk_kernel(const __grid_constant__ DecayMaps maps, const __grid_constant__ DecayArgs a) {
    using M = Map<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = smem_align1024(smem_raw);
    const uint32_t sb = smem_addr(sm);
    float *table = reinterpret_cast<float *>(sm + M::kTable), *powers = reinterpret_cast<float *>(sm + M::kPowers);
    uint64_t *bar = reinterpret_cast<uint64_t *>(sm + M::kBars);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(sm + M::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(sm + M::kMisc + 4);
    float2 *keeps = reinterpret_cast<float2 *>(sm + M::kMisc + 8);  // g^128 and g^n of the ragged chunk, as two floats

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // What this CTA walks: a pass over a whole sequence, or a segment of one (these come last, and wait for their parts alone).
    const unsigned whole_pairs = static_cast<unsigned>(a.sequences) * a.H - a.split_pairs, whole = whole_pairs * a.passes,
                   whole_too = whole + static_cast<unsigned>(a.split_pairs) * a.split_pass;
    const bool all = !PARTS && blockIdx.x < whole, cut = PARTS || blockIdx.x >= whole_too;
    const int segments = cut ? a.segments : 1;
    const unsigned first_pass = !PARTS && cut ? a.split_pass : 0,
                   passes = cut ? a.passes - first_pass : all ? a.passes : a.split_pass;
    const unsigned x = blockIdx.x - (PARTS || all ? 0 : cut ? whole_too : whole), y = x / passes;
    const unsigned nseg = PARTS ? segments - 1 : segments;
    const unsigned pi = first_pass + x % passes, segment = y % nseg, pair = y / nseg + (all ? 0 : whole_pairs);
    if (PARTS) grid_release();  // (the launch after this one has work beside it)
    const int h = pair % a.H, sequence = decay_longest_first(a, pair / a.H, reinterpret_cast<int *>(table));
    const DecayPass &ps = a.pass[pi];
    const ChunkMapsOf &mp = maps.pass[pi];
    const bool down = ps.descending != 0;
    const DecaySpan span = decay_span(a, sequence);
    const int length = static_cast<int>(span.length);
    const int chunks = (length + kC - 1) / kC, per = (chunks + segments - 1) / segments;
    const int first = min(per * static_cast<int>(segment), chunks), count = min(first + per, chunks) - first;
    const int ragged = length - (chunks - 1) * kC;  // tokens of the sequence's last chunk
    const DecayLog l2 = decay_log2(a.log_decay, h);
    // chunk r of the segment: its first token within the sequence, its tokens
    auto chunk_at = [&](int r) { return (down ? chunks - 1 - (first + r) : first + r); };
    auto begin_of = [&](int r) { return chunk_at(r) * kC; };
    auto tokens_of = [&](int r) { return chunk_at(r) == chunks - 1 ? ragged : kC; };
    // whether rows of other sequences end the chunk: one chunk of a CTA at most
    auto others_in = [&](int r) { return a.cu && tokens_of(r) < kC; };
    int *status = a.status;

    if (tid == 0) {
        for (int i = 0; i < kBars; ++i)
            mbar_init(&bar[i], i == BAR_P || i == BAR_S || i == BAR_DFREE || i == BAR_ZEROS || (i >= BAR_W && i < BAR_W + 2) ||
                                       (i >= BAR_KFREE && i < BAR_KFREE + 3)
                                   ? kWarps
                               : i == BAR_OFREE                       ? kOWarps
                               : i == BAR_VFREE || i == BAR_VFREE + 1 ? (PARTS ? 1 : 2)
                                                                      : 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0) tmem_alloc(tmem_slot, kTmemCols);
    // the factors of the segments before this one, as two floats (up to 64 products; where o's tile will lie)
    float2 *seg_keeps = reinterpret_cast<float2 *>(sm + M::kO);
    if (!PARTS && segments > 1 && tid >= 32 * kIssueWarp && tid < 32 * kIssueWarp + static_cast<int>(segment)) {
        const int g = tid - 32 * kIssueWarp, lo = min(per * g, chunks), hi = min(per * (g + 1), chunks);
        const int n = lo < hi ? (hi - lo) * kC - ((down ? lo == 0 : hi == chunks) ? kC - ragged : 0) : 0;
        seg_keeps[g] = decay_keep(l2, n);
    }
    if (segments > 1) grid_wait();  // (the segments' parts)
    if (a.cu) __syncthreads();  // (the ranks' place becomes the table's)
    if (!PARTS && tid < 256) table[tid] = tid < 127 ? 0.f : ps.p_scale * decay_power(l2, tid - 127);
    if (tid >= 256 && tid <= 256 + kC) powers[tid - 256] = ps.k_scale * decay_power(l2, tid - 256);
    if (tid >= 512 && tid < 544) reinterpret_cast<float *>(sm + M::kColumn)[tid - 512] = decay_power(l2, down ? tid - 512 : 543 - tid);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = *tmem_slot;
    const uint32_t tq = tbase + (static_cast<uint32_t>(32 * (warp & 3)) << 16);  // the warp's lane quadrant

    if (warp < kWarps) {
        // ============================================================ SP
        more_registers<kSpRegs>();
        // S^T: row `row` (of V's dimension), columns col0 .. col0 + kCols, in pairs.  (d = 64: an accumulator of 64 rows keeps
        // rows 16 q .. in lanes 32 q .., which the first four warps read, 32 columns a thread.)
        constexpr int kCols = D == 128 ? 64 : 32;
        const bool holds = D == 128 || warp < 4;
        const int row = D == 128 ? 32 * (warp & 3) + lane : 16 * (warp & 3) + (lane & 15);
        const int col0 = D == 128 ? 64 * (warp >> 2) : 32 * (lane >> 4);
        uint64_t S[kCols / 2];
        auto add = [&](const float *m, bool transposed, float2 keep) {
            const uint64_t kx = f2_make(keep.x, keep.x), ky = f2_make(keep.y, keep.y);
            const float *at = m + (transposed ? row * D + col0 : col0 * D + row);
            const int step = transposed ? 1 : D;
#pragma unroll
            for (int c = 0; c < kCols; c += 2) {
                const uint64_t f = f2_make(at[c * step], at[(c + 1) * step]);
                S[c / 2] = keep.x == 0.f ? f : f2_fma(S[c / 2], kx, f2_fma(S[c / 2], ky, f));
            }
        };
        auto put = [&](float *m) {
            if (!holds) return;
#pragma unroll
            for (int c = 0; c < kCols; c += 2) {
                const float2 f = f2_split(S[c / 2]);
                m[(col0 + c) * D + row] = f.x;
                m[(col0 + c + 1) * D + row] = f.y;
            }
        };
        auto snapshot = [&]() {  // S^T rounded to bf16, for the next chunk's Q S
            if (holds) {
#pragma unroll
                for (int c = 0; c < kCols; c += 8) {
                    const int col = col0 + c;
                    *reinterpret_cast<uint4 *>(sm + M::kS + (col >> 6) * (D * 128) + t64_chunk(row, (col & 63) >> 3)) =
                        make_uint4(bf16x2_from_f2(S[c / 2]), bf16x2_from_f2(S[c / 2 + 1]), bf16x2_from_f2(S[c / 2 + 2]),
                                   bf16x2_from_f2(S[c / 2 + 3]));
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar[BAR_S]);
        };
        auto advance = [&](int r) {  // S past chunk r
            wait_for(&bar[BAR_D], r & 1, abort_flag, status);
            tc_fence_after();
            if (r == 0) named_bar(kKeepBar, 32 * (kWarps + 1));
            const float2 keep = keeps[chunk_at(r) == chunks - 1];
            const uint64_t kx = f2_make(keep.x, keep.x), ky = f2_make(keep.y, keep.y);
#pragma unroll
            for (int c = 0; c < kCols; c += 32) {
                float d[32];
                if constexpr (D == 128)
                    tmem_ld32(tq + TM_D + col0 + c, d);
                else if (holds)
                    tmem_ld16x2_32<32>(tq + TM_D, d);
                if (c + 32 == kCols) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar[BAR_DFREE]);
                }
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    uint64_t &x = S[(c + e) / 2];
                    x = f2_fma(x, kx, f2_fma(x, ky, f2_make(d[e], d[e + 1])));
                }
            }
        };
#pragma unroll
        for (int c = 0; c < kCols / 2; ++c) S[c] = 0;
        const int64_t matrix = (static_cast<int64_t>(sequence) * a.H + h) * D * D;
        if (segments == 1 || (PARTS && segment == 0)) {
            if (ps.state_in) add(ps.state_in + matrix, ps.transposed, make_float2(0.f, 0.f));
            if (PARTS) {
                put(a.parts + decay_part(a, ps.kind, sequence, h, 0));
#pragma unroll
                for (int c = 0; c < kCols / 2; ++c) S[c] = 0;
            }
        } else if (!PARTS) {
            for (int g = 0; g <= static_cast<int>(segment); ++g)
                add(a.parts + decay_part(a, ps.kind, sequence, h, g), ps.parts_transposed, g ? seg_keeps[g - 1] : make_float2(0.f, 0.f));
        }
        const int half = warp >> 2, row0 = 32 * (warp & 3), i = row0 + lane;  // of P: column half, row
        for (int r = 0; r < count; ++r) {
            if (r) advance(r - 1);
            if (PARTS) continue;
            if (r) wait_for(&bar[BAR_O1], (r - 1) & 1, abort_flag, status);  // Q S of chunk r - 1 has read the copy
            snapshot();
            const int n = tokens_of(r);
            wait_for(&bar[BAR_A], r & 1, abort_flag, status);
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
                const int j0 = 64 * half + 32 * c;
                uint32_t p[16];
                const bool beside = (down ? j0 > row0 : j0 < row0) && (!down || j0 + 32 <= n);  // (not on the diagonal)
                const float *t = table + 127 + (down ? j0 - i : i - j0);
                if (down ? j0 + 31 < row0 || j0 >= n : j0 > row0 + 31) {  // nothing kept
#pragma unroll
                    for (int e = 0; e < 16; ++e) p[e] = 0;
                } else if (beside) {  // g^|i - j| from the row's power to the block's near edge and the column's from there
                    const float f = t[down ? 0 : -31];
                    const uint64_t f2 = f2_make(f, f);
                    const ulonglong2 *column = reinterpret_cast<const ulonglong2 *>(sm + M::kColumn);
                    float v[32];
                    tmem_ld32(tq + TM_A + j0, v);
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const ulonglong2 cc = column[e / 4];
                        p[e / 2] = bf16x2_from_f2(f2_mul(f2_mul(f2_make(v[e], v[e + 1]), cc.x), f2));
                        p[e / 2 + 1] = bf16x2_from_f2(f2_mul(f2_mul(f2_make(v[e + 2], v[e + 3]), cc.y), f2));
                    }
                } else {
                    float v[32];
                    tmem_ld32(tq + TM_A + j0, v);
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
        }
        if (count) advance(count - 1);
        if (PARTS)
            put(a.parts + decay_part(a, ps.kind, sequence, h, segment + 1));
        else if (ps.state_out && static_cast<int>(segment) == segments - 1)
            put(ps.state_out + matrix);
    } else if (warp < kOWarp0) {
        // ============================================================ W
        fewer_registers<kWRegs>();
        const int wt = tid - 32 * kWWarp0;
        // this thread's 16-byte chunk of rows wr + kRows k of a quarter
        constexpr int kWide = D / 8, kRows = 32 * kWarps / kWide;
        const int wc = wt % kWide, wr = wt / kWide;
        const uint8_t *k_mine = sm + M::kK + (wc >> 3) * M::kKBlock + t64_chunk(wr, wc & 7);
        uint8_t *w_mine = sm + M::kW + (wc >> 3) * M::kWBlock + t64_chunk(wr, wc & 7);
        Ring ring;
        for (int r = 0; r < count; ++r) {
            const uint32_t par = r & 1;
            const int n = tokens_of(r);
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                const int slot = q & 1;
                if (!(q & 1)) wait_for(&bar[BAR_K + ring.slot], ring.parity, abort_flag, status);
                if (r || q > 1) wait_for(&bar[BAR_WFREE + slot], q > 1 ? 0 : 1, abort_flag, status);
                const uint8_t *k_from = k_mine + ring.slot * M::kHBlock + 32 * 128 * (q & 1);
                uint8_t *w_to = w_mine + slot * M::kWSlot;
#pragma unroll
                for (int k = 0; k < 32 / kRows; ++k) {
                    const int t = 32 * q + wr + kRows * k;  // (kRows rows on: the same place of the swizzle)
                    const uint4 u = *reinterpret_cast<const uint4 *>(k_from + kRows * 128 * k);
                    uint4 hi = make_uint4(0, 0, 0, 0), mid = hi, lo = hi;
                    if (t < n) {
                        const float w = powers[down ? t + 1 : n - 1 - t];
                        const uint64_t ww = f2_make(w, w);
                        split<TERMS>(f2_mul(f2_from_bf16x2(u.x), ww), hi.x, mid.x, lo.x);
                        split<TERMS>(f2_mul(f2_from_bf16x2(u.y), ww), hi.y, mid.y, lo.y);
                        split<TERMS>(f2_mul(f2_from_bf16x2(u.z), ww), hi.z, mid.z, lo.z);
                        split<TERMS>(f2_mul(f2_from_bf16x2(u.w), ww), hi.w, mid.w, lo.w);
                    }
                    uint8_t *to = w_to + kRows * 128 * k;
                    *reinterpret_cast<uint4 *>(to) = hi;
                    *reinterpret_cast<uint4 *>(to + M::kWTerm) = mid;
                    if (TERMS == 3) *reinterpret_cast<uint4 *>(to + 2 * M::kWTerm) = lo;
                }
                if (q == 0 && others_in(r)) {  // zeros in V
                    for (int j = 0; j < 2; ++j) {
                        wait_for(&bar[BAR_V + j], par, abort_flag, status);
                        for (int t = max(n - 64 * j, 0) + wr; t < 64; t += kRows)
                            *reinterpret_cast<uint4 *>(sm + M::kV + j * M::kHalf + (wc >> 3) * M::kHBlock +
                                                       t64_chunk(t, wc & 7)) = make_uint4(0, 0, 0, 0);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bar[BAR_W + slot]);
                    if (q == 0 && others_in(r)) mbar_arrive(&bar[BAR_ZEROS]);
                    if (q & 1) mbar_arrive(&bar[BAR_KFREE + ring.slot]);
                }
                if (q & 1) ring.next();
            }
        }
    } else if (warp < kIssueWarp) {
        // ============================================================ O
        fewer_registers<kORegs>();
        const int i = 32 * (warp & 3) + lane;
        const bool storer = tid == 32 * kOWarp0, fp32 = SUMS && ps.o_fp32;
        const float near = decay_power(l2, i + 1) * ps.s_scale;  // ascending, or a full chunk's mirror image below
        const float far = decay_power(l2, kC - 1 - i) * ps.s_scale;
        for (int r = 0; r < (PARTS ? 0 : count); ++r) {
            const int n = tokens_of(r);
            const float fac = down ? (n == kC ? far : i < n ? decay_power(l2, n - 1 - i) * ps.s_scale : 0.f) : near;
            const int64_t at = span.b * ps.o_batch + (span.begin + begin_of(r) + i) * ps.o_token + h * ps.o_head;
            const bool by_rows = others_in(r);
            auto wait_tile = [&]() {  // the tile has been read
                if (storer) tma_store_wait_read();
                named_bar(kOutBar, 32 * kOWarps);
            };
            auto store_tile = [&](int column, int columns) {
                fence_proxy_async_smem();
                named_bar(kOutBar, 32 * kOWarps);
                if (storer) {
                    for (int c = 0; c < columns; c += 128 / (fp32 ? 4 : 2))
                        tma_store_4d(&mp.o, sm + M::kO + c * (fp32 ? M::kBlock / 32 : M::kBlock / 64), column + c, h,
                                     static_cast<int>(span.begin) + begin_of(r), static_cast<int>(span.b));
                    tma_store_commit();
                }
            };
            if (!by_rows) wait_tile();
            wait_for(&bar[BAR_O1], r & 1, abort_flag, status);
            wait_for(&bar[BAR_O2], r & 1, abort_flag, status);
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
                if (!by_rows && fp32 && c && !(c & 3)) wait_tile();  // (in fp32 64 columns at a time)
                float u[16], w[16];
                tmem_ld16_two(tq + TM_O1 + 16 * c, tq + TM_O2 + 16 * c, u, w);
                if (c == D / 16 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar[BAR_OFREE]);
                }
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 f = f2_split(f2_fma(f2_make(u[e], u[e + 1]), f2_make(fac, fac), f2_make(w[e], w[e + 1])));
                    u[e] = f.x;
                    u[e + 1] = f.y;
                }
                if (fp32) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 four = make_float4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                        if (!by_rows)
                            *reinterpret_cast<float4 *>(sm + M::kO + ((c >> 1) & 1) * M::kBlock +
                                                        t64_chunk(i, 4 * (c & 1) + e / 4)) = four;
                        else if (i < n)
                            *reinterpret_cast<float4 *>(static_cast<float *>(ps.o) + at + 16 * c + e) = four;
                    }
                    if (!by_rows && (c & 3) == 3) store_tile(16 * (c - 3), 64);
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                    const uint4 packed = make_uint4(pack_bf16(u[e], u[e + 1]), pack_bf16(u[e + 2], u[e + 3]),
                                                    pack_bf16(u[e + 4], u[e + 5]), pack_bf16(u[e + 6], u[e + 7]));
                    if (!by_rows)
                        *reinterpret_cast<uint4 *>(sm + M::kO + (c >> 2) * M::kBlock + t64_chunk(i, 2 * (c & 3) + e / 8)) = packed;
                    else if (i < n)
                        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(ps.o) + at + 16 * c + e) = packed;
                }
            }
            if (!by_rows && !fp32) store_tile(0, D);
        }
        if (storer) tma_store_wait_all();
    } else {
        fewer_registers<kOtherRegs>();
        if (warp == kIssueWarp && elect_one()) {
            // ======================================================== ISSUE: Q K^T, Q S, P V
            constexpr uint32_t kQK = make_idesc(kC, kC, 0, 0), kQKHalf = make_idesc(kC, 64, 0, 0), kQS = make_idesc(kC, D, 0, 0),
                               kPV = make_idesc(kC, D, 0, 1);
            Ring ring;
            for (int r = 0; r < (PARTS ? 0 : count); ++r) {
                const uint32_t par = r & 1, before = par ^ 1;
                wait_for(&bar[BAR_Q], par, abort_flag, status);
                if (r) wait_for(&bar[BAR_O2], before, abort_flag, status);  // P V has read P, which lies in A
                uint32_t kh[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    wait_for(&bar[BAR_K + ring.slot], ring.parity, abort_flag, status);
                    kh[j] = sb + M::kK + ring.slot * M::kHBlock;
                    ring.next();
                }
                tc_fence_after();
                if (kh[1] > kh[0]) {  // the halves are neighbours
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_bf16(tbase + TM_A, desc_kmajor(sb + M::kQ + (k >> 2) * M::kBlock, k & 3),
                                 desc_kmajor(kh[0] + (k >> 2) * M::kKBlock, k & 3), kQK, k > 0);
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            mma_bf16(tbase + TM_A + 64 * j, desc_kmajor(sb + M::kQ + (k >> 2) * M::kBlock, k & 3),
                                     desc_kmajor(kh[j] + (k >> 2) * M::kKBlock, k & 3), kQKHalf, k > 0);
                }
                mma_commit(&bar[BAR_A]);
                wait_for(&bar[BAR_S], par, abort_flag, status);
                if (r) wait_for(&bar[BAR_OFREE], before, abort_flag, status);
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_bf16(tbase + TM_O1, desc_kmajor(sb + M::kQ + (k >> 2) * M::kBlock, k & 3),
                             desc_kmajor(sb + M::kS + (k >> 2) * (D * 128), k & 3), kQS, k > 0);
                mma_commit(&bar[BAR_O1]);
                for (int j = 0; j < 2; ++j) wait_for(&bar[BAR_V + j], par, abort_flag, status);
                if (others_in(r)) wait_for(&bar[BAR_ZEROS], 0, abort_flag, status);
                wait_for(&bar[BAR_P], par, abort_flag, status);
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < kC / 16; ++k)
                    mma_bf16_ts(tbase + TM_O2, tbase + TM_A + 64 * (k >> 2) + 8 * (k & 3),
                                desc_mnmajor(sb + M::kV + (k >> 2) * M::kHalf, M::kHBlock, k & 3), kPV, k > 0);
                mma_commit(&bar[BAR_O2]);
                for (int j = 0; j < 2; ++j) mma_commit(&bar[BAR_VFREE + j]);
            }
        } else if (warp == kIssueWWarp && elect_one()) {
            // ======================================================== ISSUE: V^T W, beside the other products
            constexpr uint32_t kWV = make_idesc(D, D, 1, 1);
            for (int r = 0; r < count; ++r) {
                const uint32_t par = r & 1, before = par ^ 1;
                if (r) wait_for(&bar[BAR_DFREE], before, abort_flag, status);
#pragma unroll 1
                for (int q = 0; q < 4; ++q) {
                    const int slot = q & 1, half = q >> 1;
                    if (!slot) wait_for(&bar[BAR_V + half], par, abort_flag, status);
                    wait_for(&bar[BAR_W + slot], half, abort_flag, status);
                    tc_fence_after();
                    const uint32_t w = sb + M::kW + slot * M::kWSlot, v = sb + M::kV + half * M::kHalf;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int t = TERMS - 1; t >= 0; --t)  // the small terms first
                            mma_bf16(tbase + TM_D, desc_mnmajor(v, M::kHBlock, 2 * slot + k),
                                     desc_mnmajor(w + t * M::kWTerm, M::kWBlock, k), kWV, q > 0 || k > 0 || t < TERMS - 1);
                    mma_commit(&bar[BAR_WFREE + slot]);
                    if (slot) mma_commit(&bar[BAR_VFREE + half]);
                }
                mma_commit(&bar[BAR_D]);
            }
        } else if (warp == kLoadWarp && elect_one()) {
            // ======================================================== LOAD
            const int hq = h / ps.q.share, hk = h / ps.k.share, hv = h / ps.v.share, b = static_cast<int>(span.b);
            auto load = [&](const CUtensorMap *map, uint32_t to, uint32_t block, uint32_t apart, uint64_t *full, int head, int token) {
                mbar_arrive_expect_tx(full, block * M::kBlocks);
#pragma unroll
                for (uint32_t c = 0; c < M::kBlocks; ++c) tma_load_4d(sm + to + c * apart, map, full, 64 * c, head, token, b);
            };
            Ring ring;
            auto load_k = [&](int half, int token) {
                if (half > 2) wait_for(&bar[BAR_KFREE + ring.slot], ring.parity ^ 1, abort_flag, status);
                load(&mp.k, M::kK + ring.slot * M::kHBlock, M::kHBlock, M::kKBlock, &bar[BAR_K + ring.slot], hk, token);
                ring.next();
            };
            tma_prefetch_desc(&mp.k);
            tma_prefetch_desc(&mp.v);
            if (!PARTS) tma_prefetch_desc(&mp.q);
            // a tile of the next chunk into L2, behind the load of its place in this chunk: what is under way then covers HBM's latency
            auto ahead = [&](int r, const CUtensorMap *map, int head, int offset) {
                if (r + kAhead >= count) return;
                const int next = static_cast<int>(span.begin) + begin_of(r + kAhead) + offset;
#pragma unroll
                for (uint32_t c = 0; c < M::kBlocks; ++c) tma_prefetch_l2_4d(map, 64 * c, head, next, b);
            };
            for (int r = 0; r < count; ++r) {
                const uint32_t before = (r & 1) ^ 1;
                const int token = static_cast<int>(span.begin) + begin_of(r);
                load_k(2 * r, token);  // (Q K^T of chunk r - 2 was waited for with the half before this one)
                ahead(r, &mp.k, hk, 0);
                if (!PARTS && r) wait_for(&bar[BAR_A], before, abort_flag, status);
                load_k(2 * r + 1, token + 64);
                ahead(r, &mp.k, hk, 64);
                if (!PARTS) {
                    if (r) wait_for(&bar[BAR_O1], before, abort_flag, status);
                    load(&mp.q, M::kQ, M::kBlock, M::kBlock, &bar[BAR_Q], hq, token);
                    ahead(r, &mp.q, hq, 0);
                }
                for (int j = 0; j < 2; ++j) {
                    if (r) wait_for(&bar[BAR_VFREE + j], before, abort_flag, status);
                    load(&mp.v, M::kV + j * M::kHalf, M::kHBlock, M::kHBlock, &bar[BAR_V + j], hv, token + 64 * j);
                    ahead(r, &mp.v, hv, 64 * j);
                }
            }
            // no CTA leaves before its copies have landed (after a wait that ran out)
            if (count > 0) {
                const uint32_t last = (count - 1) & 1;
                if (!PARTS) mbar_drain(&bar[BAR_Q], last);
                for (int j = 0; j < 2; ++j) mbar_drain(&bar[BAR_V + j], last);
                for (int half = max(0, 2 * count - 3); half < 2 * count; ++half) mbar_drain(&bar[BAR_K + half % 3], (half / 3) & 1);
            }
        } else if (warp == kKeepWarp && count > 0) {
            // ======================================================== the powers in 64 bits, a microsecond that SP needs not wait for
            if (lane < 2) keeps[lane] = decay_keep(l2, lane ? ragged : kC);
            __syncwarp();
            named_bar_arrive(kKeepBar, 32 * (kWarps + 1));
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tbase, kTmemCols);
}

template <int D, bool PARTS, int TERMS, bool SUMS> cudaError_t launch(const DecayMaps &m, const DecayArgs &a, cudaStream_t s) {
    constexpr int kBytes = Map<D>::kBytes;
    cudaError_t e = allow_shared<decay_chunk_kernel<D, PARTS, TERMS, SUMS>>(kBytes);
    if (e != cudaSuccess) return e;
    const int64_t pairs = static_cast<int64_t>(a.H) * a.sequences, split = a.split_pairs;
    const int64_t grid = PARTS ? split * (a.segments - 1) * a.passes
                               : (pairs - split) * a.passes + split * (a.split_pass + (a.passes - a.split_pass) * a.segments);
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    if (!PARTS && split)
        return launch_after(decay_chunk_kernel<D, PARTS, TERMS, SUMS>, static_cast<unsigned>(grid), kThreads, kBytes, s, m, a);
    decay_chunk_kernel<D, PARTS, TERMS, SUMS><<<static_cast<unsigned>(grid), kThreads, kBytes, s>>>(m, a);
    return cudaGetLastError();
}

template <int D, int TERMS> cudaError_t launch_any(const DecayMaps &m, const DecayArgs &a, cudaStream_t s) {
    if (a.parts_only) return launch<D, true, TERMS, false>(m, a, s);
    for (int i = 0; i < a.passes; ++i)
        if (a.pass[i].o_fp32) return launch<D, false, TERMS, true>(m, a, s);
    return launch<D, false, TERMS, false>(m, a, s);
}

}  // namespace

cudaError_t launch_decay_chunks(const DecayArgs &a, int64_t B, cudaStream_t s) {
    DecayMaps m;
    const DecayView *seen[9];
    int tokens[9];
    const CUtensorMap *made[9];
    int count = 0;
    for (int i = 0; i < a.passes; ++i) {
        const DecayView *views[3] = {&a.pass[i].q, &a.pass[i].k, &a.pass[i].v};
        CUtensorMap *to[3] = {&m.pass[i].q, &m.pass[i].k, &m.pass[i].v};
        for (int j = 0; j < 3; ++j) {
            const DecayView &x = *views[j];
            int k = 0;  // (the gradients' passes read the same tensors)
            const int box = j ? 64 : kC;
            while (k < count && (tokens[k] != box || !(*seen[k] == x))) ++k;
            if (k < count) {
                *to[j] = *made[k];
                continue;
            }
            if (!make_heads_map(to[j], x.p, 2, B, a.T, a.H / x.share, a.d, x.batch, x.token, x.head, box))
                return cudaErrorInvalidValue;
            seen[count] = &x;
            tokens[count] = box;
            made[count++] = to[j];
        }
        const DecayPass &ps = a.pass[i];
        if (a.parts_only)
            m.pass[i].o = m.pass[i].q;  // (not used)
        else if (!make_heads_map(&m.pass[i].o, ps.o, ps.o_fp32 ? 4 : 2, B, a.T, a.H, a.d, ps.o_batch, ps.o_token, ps.o_head, kC))
            return cudaErrorInvalidValue;
    }
    if (a.exact_state) return a.d == 128 ? launch_any<128, 3>(m, a, s) : launch_any<64, 3>(m, a, s);
    return a.d == 128 ? launch_any<128, 2>(m, a, s) : launch_any<64, 2>(m, a, s);
}

}  // namespace ccq

// ccq_embed.cu -- embedding lookup with scaling and the gradient of its table (ccq_ops.h).
//
// Lookup: out[i] = scale * table[ids[i]], a copy of n rows; bound by HBM (each row read once and
// written once).
//
// Gradient: dtable[r] = scale * sum of dout[i] over the i with ids[i] = r.  Each row of dout is read
// once and each row of dtable written once; no sum depends on the order of atomics:
//   1. embed_sort_kernel: a stable radix sort of (id, i), one cluster of 8 CTAs, all passes in one launch.
//      It also marks where each piece of the path below begins.
//   2. embed_sum_kernel: the sorted entries and the rows' ends form one path of n + rows steps (the
//      entries of row 0, its end, the entries of row 1, its end, ...).  The path is cut into pieces of
//      kPiece steps, so frequent ids and empty rows cost the same everywhere.  A warp takes a piece of a
//      column slice: it adds the entries and writes a row at its end.  What it holds of a row that began in
//      an earlier piece, or ends in a later one, goes to the workspace.
//   3. embed_join_kernel: adds the parts of the rows that span pieces, in order.
#include <algorithm>

#include "ccq_ops.cuh"

namespace ccq {
namespace {

// ---------------------------------------------------------------- lookup

constexpr int kLookupThreads = 256;
constexpr int kLookupRows = 4;  // rows in flight per thread

// Threads (tx, ty): tx along a row, ty rows at a time, kLookupRows of them apart.
template <typename T, int N>
__global__ void __launch_bounds__(kLookupThreads) embed_kernel(const T *__restrict__ table, int64_t table_stride,
                                                               const void *__restrict__ ids, int id_bytes, int64_t n,
                                                               int64_t rows, int packs, float scale, T *out,
                                                               int64_t out_stride, int *status) {
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * kLookupRows) * blockDim.y + threadIdx.y;
    int64_t id[kLookupRows];
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
        const int64_t i = first + r * blockDim.y;
        id[r] = i < n ? load_index(ids, id_bytes, i) : -1;
        if (i < n && (id[r] < 0 || id[r] >= rows)) {
            id[r] = -1;
            if (threadIdx.x == 0 && blockIdx.y == 0) note_index(status);
        }
    }
    for (int c = blockIdx.y * blockDim.x + threadIdx.x; c < packs; c += gridDim.y * blockDim.x) {
        Pack<T, N> v[kLookupRows];
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
            v[r].raw = {};
            if (id[r] >= 0) v[r] = load_plain<T, N>(table + id[r] * table_stride + static_cast<int64_t>(c) * N);
        }
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
            const int64_t i = first + r * blockDim.y;
            if (i >= n) continue;
            float f[N];
            unpack(v[r], f);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] *= scale;
            pack(f, v[r]);
            store_stream<T, N>(out + i * out_stride + static_cast<int64_t>(c) * N, v[r]);
        }
    }
}

template <typename T, int N>
cudaError_t launch_embed(const void *table, int64_t table_stride, const void *ids, int id_bytes, int64_t n,
                         int64_t rows, int width, float scale, void *out, int64_t out_stride, cudaStream_t s) {
    const int packs = width / N;
    int tx = 32;
    while (tx < kLookupThreads && tx < packs) tx *= 2;
    const int ty = kLookupThreads / tx;
    const dim3 grid(static_cast<unsigned>((n + ty * kLookupRows - 1) / (ty * kLookupRows)), 1);
    embed_kernel<T, N><<<grid, dim3(tx, ty), 0, s>>>(
        static_cast<const T *>(table), table_stride, ids, id_bytes, n, rows, packs, scale, static_cast<T *>(out),
        out_stride, device_status_word());
    return cudaGetLastError();
}

// ---------------------------------------------------------------- sort

constexpr int kSortCtas = 8;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxDigit = 10;  // bits of a pass
constexpr int kHeld = 4;       // entries a lane keeps in registers; with more, a pass reads them twice
constexpr int kPiece = 32;     // path steps of a piece

struct SortArgs {
    const void *ids;
    int id_bytes;
    int n;
    int64_t rows, padding;
    int passes, digit;
    uint32_t *key[2];
    uint32_t *pos[2];
    int *piece_start;  // [pieces + 1]: entries before each piece's first step
    int pieces;
    int *joins;        // count, then the pieces that end a row from an earlier one (embed_sum_kernel)
    int *status;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ void cluster_store(uint32_t *p, int cta, uint32_t v) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(cta));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

// Every warp owns a contiguous range of the entries, warps and CTAs in order, so ranks within a warp, sums over
// the warps before it and over the CTAs before that keep equal digits in order.  Invalid and padding ids get the
// key `rows`, behind every row.  All passes run in one launch: n = 16384 takes two and about a sixth of the whole call.
__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) embed_sort_kernel(SortArgs a) {
    extern __shared__ uint32_t smem[];
    const int bins = 1 << a.digit;
    uint32_t *counts = smem;                     // [kSortWarps][bins]: a warp's entries, then its first slot of each bin
    uint32_t *totals = smem + kSortWarps * bins;  // [kSortCtas][bins]: every CTA's entries
    __shared__ uint32_t scan[kSortWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const int per = ((a.n + kSortCtas * kSortWarps - 1) / (kSortCtas * kSortWarps) + 31) & ~31;
    const int64_t lo64 = static_cast<int64_t>(cta * kSortWarps + warp) * per;
    const int lo = static_cast<int>(lo64 < a.n ? lo64 : a.n);
    const int hi = lo + (a.n - lo < per ? a.n - lo : per);
    const bool held = per <= 32 * kHeld;
    uint32_t *mine = counts + warp * bins;
    if (cta == 0 && tid == 0) a.joins[0] = 0;
    cluster_sync();  // every CTA runs before its shared memory is written
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit;
        const uint32_t *key = a.key[(pass + 1) & 1], *pos = a.pos[(pass + 1) & 1];
        uint32_t *key_out = a.key[pass & 1], *pos_out = a.pos[pass & 1];
        auto key_from = [&](int64_t id) -> uint32_t {
            if (id < 0 || id >= a.rows) {
                note_index(a.status);
                return static_cast<uint32_t>(a.rows);
            }
            return static_cast<uint32_t>(id == a.padding ? a.rows : id);
        };
        auto key_of = [&](int i) -> uint32_t { return pass ? key[i] : key_from(load_index(a.ids, a.id_bytes, i)); };
        uint32_t k[kHeld], p[kHeld], slot[kHeld];
        if (held && pass) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                const int i = lo + q * 32 + lane;
                k[q] = i < hi ? key[i] : 0;
                p[q] = i < hi ? pos[i] : 0;
            }
        } else if (held) {
            int64_t id[kHeld];
            if (a.id_bytes == 8) {
#pragma unroll
                for (int q = 0; q < kHeld; ++q) id[q] = lo + q * 32 + lane < hi ? static_cast<const int64_t *>(a.ids)[lo + q * 32 + lane] : 0;
            } else {
#pragma unroll
                for (int q = 0; q < kHeld; ++q) id[q] = lo + q * 32 + lane < hi ? static_cast<const int32_t *>(a.ids)[lo + q * 32 + lane] : 0;
            }
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                p[q] = static_cast<uint32_t>(lo + q * 32 + lane);
                k[q] = key_from(id[q]);
            }
        }
        for (int i = tid; i < kSortWarps * bins; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        // an entry's place among its warp's of the same digit
        auto place = [&](uint32_t key_, bool live) -> uint32_t {
            const uint32_t d = live ? (key_ >> shift) & (bins - 1) : ~0u;
            const uint32_t same = __match_any_sync(~0u, d);
            const int rank = __popc(same & ((1u << lane) - 1));
            uint32_t at = 0;
            if (live) at = mine[d] + rank;
            __syncwarp();
            if (live && rank == 0) mine[d] += __popc(same);
            __syncwarp();
            return at;
        };
        if (held) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q)
                if (lo + q * 32 < hi) slot[q] = place(k[q], lo + q * 32 + lane < hi);
        } else {
            for (int i0 = lo; i0 < hi; i0 += 32) place(i0 + lane < hi ? key_of(i0 + lane) : 0, i0 + lane < hi);
        }
        __syncthreads();
        // this CTA's entries of every bin to all CTAs
        if (tid < bins) {
            uint32_t sum = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) sum += counts[w * bins + tid];
            for (int c = 0; c < kSortCtas; ++c) cluster_store(&totals[cta * bins + tid], c, sum);
        }
        cluster_sync();
        uint32_t all = 0, before = 0;
        if (tid < bins)
            for (int c = 0; c < kSortCtas; ++c) {
                const uint32_t t = totals[c * bins + tid];
                if (c < cta) before += t;
                all += t;
            }
        // exclusive scan of `all` over the bins
        uint32_t inc = all;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 31) scan[warp] = inc;
        __syncthreads();
        if (tid < bins) {
            uint32_t base = inc - all + before;
            for (int w = 0; w < warp; ++w) base += scan[w];
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = counts[w * bins + tid];
                counts[w * bins + tid] = base;
                base += c;
            }
        }
        __syncthreads();
        if (held) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                if (lo + q * 32 + lane >= hi) continue;
                const uint32_t at = slot[q] + mine[(k[q] >> shift) & (bins - 1)];
                key_out[at] = k[q];
                pos_out[at] = p[q];
            }
        } else {
            for (int i0 = lo; i0 < hi; i0 += 32) {
                const int i = i0 + lane;
                const bool live = i < hi;
                const uint32_t kk = live ? key_of(i) : 0, at = place(kk, live);
                if (live) {
                    key_out[at] = kk;
                    pos_out[at] = pass ? pos[i] : static_cast<uint32_t>(i);
                }
            }
        }
        cluster_sync();  // the next pass reads what the other CTAs wrote, and `totals` may be written again
    }
    // Entry i is step i + key[i] of the path, so it is the first of the pieces that start after entry i - 1's step and
    // not after its own; those that start after the last entry's have none.
    const uint32_t *key = a.key[(a.passes + 1) & 1];
    for (int i0 = (cta * kSortWarps + warp) * 32; i0 <= a.n; i0 += kSortCtas * kSortThreads) {
        const int i = i0 + lane;
        int64_t first = 0, last = -1;
        if (i <= a.n) {
            first = i ? (static_cast<int64_t>(i - 1) + key[i - 1]) / kPiece + 1 : 0;
            last = i < a.n ? (static_cast<int64_t>(i) + key[i]) / kPiece : a.pieces;
        }
        // long gaps are filled by the whole warp
        uint32_t wide = __ballot_sync(~0u, last - first >= 4);
        if (last - first < 4)
            for (int64_t q = first; q <= last; ++q) a.piece_start[q] = i;
        while (wide) {
            const int src = __ffs(wide) - 1;
            wide &= wide - 1;
            const int64_t f = __shfl_sync(~0u, first, src), l = __shfl_sync(~0u, last, src);
            for (int64_t q = f + lane; q <= l; q += 32) a.piece_start[q] = i0 + src;
        }
    }
}

// ---------------------------------------------------------------- sums

struct SumArgs {
    const void *dout;
    int64_t dout_stride;
    const uint32_t *key, *pos;  // sorted entries
    const int *piece_start;
    int *joins;
    int n, rows, width, packs;
    float scale;
    void *dtable;
    int64_t dtable_stride;
    float *part;  // [pieces][2][width]: what a piece holds of a row from before it, and of a row it leaves open
    int pieces;
};

constexpr int kSumThreads = 256;

template <typename T, typename O, int N> __global__ void __launch_bounds__(kSumThreads, 4) embed_sum_kernel(SumArgs a) {
    constexpr int kFlight = N >= 8 ? 4 : 8;  // entries whose loads are under way at once
    grid_wait();
    const int lane = threadIdx.x & 31;
    const int slices = (a.packs + 31) / 32;
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kSumThreads / 32) + (threadIdx.x >> 5);
    const int64_t piece = warp / slices;
    if (piece >= a.pieces) return;
    const int slice = static_cast<int>(warp - piece * slices);
    const int c = slice * 32 + lane;
    const bool live = c < a.packs;
    const T *dout = static_cast<const T *>(a.dout) + static_cast<int64_t>(c) * N;
    O *dtable = static_cast<O *>(a.dtable) + static_cast<int64_t>(c) * N;
    const int64_t step0 = piece * kPiece, step1 = step0 + kPiece;
    const int last = a.pieces;
    const int before = piece > 0 ? a.piece_start[piece - 1] : 0;
    int i0 = a.piece_start[piece];
    const int i1 = a.piece_start[piece + 1], i2 = a.piece_start[piece + 2 < last ? piece + 2 : last];
    int v = static_cast<int>(step0 - i0 < a.rows ? step0 - i0 : a.rows);
    int v1 = static_cast<int>(step1 - i1 < a.rows ? step1 - i1 : a.rows);
    const int64_t v2 = piece + 2 < last ? step1 + kPiece - i2 : a.rows;  // rows that end before the piece after the next
    // the piece's entries and those of the next, one a lane (there are at most kPiece each), and the entry before each
    uint32_t key = ~0u, pos = 0, key2 = ~0u, pos2 = 0;
    if (i0 + lane < i1) {
        key = a.key[i0 + lane];
        pos = a.pos[i0 + lane];
    }
    if (i1 + lane < i2) {
        key2 = a.key[i1 + lane];
        pos2 = a.pos[i1 + lane];
    }
    const uint32_t before0 = i0 > 0 ? a.key[i0 - 1] : ~0u, before1 = before > 0 ? a.key[before - 1] : ~0u;
    // the sum in hand belongs to a row with entries before this piece
    bool head = v < a.rows && before0 == static_cast<uint32_t>(v);
    int skip = 0;  // entries that the piece before takes
    if (head && before1 != static_cast<uint32_t>(v) && v < v1) {
        // the row began in the piece before and ends here: that piece finishes it
        skip = __popc(__ballot_sync(~0u, key == static_cast<uint32_t>(v)));
        head = false;
        ++v;
    }
    // the row left open at the end of this piece ends in the next one: finished here, if it began here
    int more = 0;
    const uint32_t open = static_cast<uint32_t>(v1);
    if (v1 < a.rows && v1 < v2 && (v < v1 || !head)) {
        const uint32_t last_key = i1 > 0 ? a.key[i1 - 1] : ~0u;
        if (last_key == open && i1 > i0 + skip) {
            more = __popc(__ballot_sync(~0u, key2 == open));
            ++v1;
        }
    }
    if (head && v < v1 && slice == 0 && lane == 0) a.joins[1 + atomicAdd(a.joins, 1)] = static_cast<int>(piece);
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    auto end_row = [&] {
        if (live) {
            if (head) {
                float *to = a.part + piece * 2 * a.width + c * N;
#pragma unroll
                for (int e = 0; e < N; ++e) to[e] = acc[e];
            } else {
                Pack<O, N> o;
                float f[N];
#pragma unroll
                for (int e = 0; e < N; ++e) f[e] = acc[e] * a.scale;
                pack(f, o);
                store_stream<O, N>(dtable + static_cast<int64_t>(v) * a.dtable_stride, o);
            }
        }
        head = false;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.f;
        ++v;
    };
    // entries behind the last row's (invalid and padding ids) are left out
    const int own = __popc(__ballot_sync(~0u, key < static_cast<uint32_t>(a.rows))), count = own + more;
    for (int q0 = skip; q0 < count; q0 += kFlight) {
        Pack<T, N> x[kFlight];
#pragma unroll
        for (int q = 0; q < kFlight; ++q) {
            const int at = q0 + q;
            const uint32_t row = at < own ? __shfl_sync(~0u, pos, at & 31) : __shfl_sync(~0u, pos2, (at - own) & 31);
            x[q].raw = {};
            if (live && at < count) x[q] = load_stream<T, N>(dout + static_cast<int64_t>(row) * a.dout_stride);
        }
#pragma unroll
        for (int q = 0; q < kFlight; ++q) {
            const int at = q0 + q;
            if (at >= count) break;
            const uint32_t k = at < own ? __shfl_sync(~0u, key, at & 31) : open;
            while (v < static_cast<int>(k)) end_row();
            float f[N];
            unpack(x[q], f);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += f[e];
        }
    }
    while (v < v1) end_row();
    if (live && v < a.rows) {
        float *to = a.part + (piece * 2 + 1) * a.width + c * N;
#pragma unroll
        for (int e = 0; e < N; ++e) to[e] = acc[e];
    }
}

// The rows that span pieces: the parts of the pieces before the one that ends the row, then that one's.  A CTA takes 64
// columns of a row, 16 threads 4 columns each, in 16 strided sums over the pieces that are then added in order.
constexpr int kJoinColumns = 64;
constexpr int kJoinCtas = 608;
template <typename O> __global__ void __launch_bounds__(kSumThreads) embed_join_kernel(SumArgs a) {
    __shared__ float sums[16][kJoinColumns + 1];
    grid_wait();
    const int count = a.joins[0], chunks = (a.width + kJoinColumns - 1) / kJoinColumns;
    const int column = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
    for (int64_t job = blockIdx.x; job < static_cast<int64_t>(count) * chunks; job += gridDim.x) {
        const int64_t piece = a.joins[1 + job / chunks];
        const int c0 = static_cast<int>(job % chunks) * kJoinColumns;
        const int v = static_cast<int>(piece * kPiece - a.piece_start[piece]);
        // the first piece with entries of row v: its first entry's, at step lo + v; a warp tries 32 places at a time
        int lo = 0, hi = a.piece_start[piece];
        while (lo < hi) {
            const int stride = (hi - lo + 31) / 32, at = lo + (threadIdx.x & 31) * stride;
            const uint32_t below = __ballot_sync(~0u, at < hi && a.key[at < hi ? at : hi - 1] < static_cast<uint32_t>(v));
            if (!below) break;
            const int top = __popc(below) - 1;  // the last place whose key is below v
            const int from = lo + top * stride;
            hi = from + stride < hi ? from + stride : hi;
            lo = from + 1;
        }
        const int64_t first = (static_cast<int64_t>(lo) + v) / kPiece;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int64_t p = first + group; p <= piece; p += 16) {
            const float *from = a.part + (p * 2 + (p < piece)) * a.width + c0 + column;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c0 + column + e < a.width) s[e] += from[e];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[group][column + e] = s[e];
        __syncthreads();
        if (threadIdx.x < kJoinColumns && c0 + static_cast<int>(threadIdx.x) < a.width) {
            float t = 0.f;
#pragma unroll
            for (int g = 0; g < 16; ++g) t += sums[g][threadIdx.x];
            static_cast<O *>(a.dtable)[static_cast<int64_t>(v) * a.dtable_stride + c0 + threadIdx.x] = from_f32<O>(t * a.scale);
        }
    }
}

template <typename T, typename O, int N> cudaError_t launch_sum(SumArgs a, cudaStream_t s) {
    a.packs = a.width / N;
    const int64_t warps = static_cast<int64_t>(a.pieces) * ((a.packs + 31) / 32);
    const int per = kSumThreads / 32;
    cudaError_t e = launch_after(embed_sum_kernel<T, O, N>, static_cast<unsigned>((warps + per - 1) / per), kSumThreads,
                                 0, s, a);
    if (e != cudaSuccess) return e;
    return launch_after(embed_join_kernel<O>, kJoinCtas, kSumThreads, 0, s, a);
}

int key_bits(int64_t rows) {  // keys 0 .. rows
    int b = 1;
    while ((static_cast<int64_t>(1) << b) <= rows) ++b;
    return b;
}

int64_t piece_count(int64_t n, int64_t rows) { return (n + rows + kPiece - 1) / kPiece; }

size_t round16(size_t x) { return (x + 15) & ~static_cast<size_t>(15); }

size_t grad_workspace(int64_t n, int64_t rows, int width) {
    const size_t pieces = static_cast<size_t>(piece_count(n, rows));
    return 4 * round16(static_cast<size_t>(n) * 4) + 2 * round16((pieces + 1) * 4) +
           round16(pieces * 2 * width * sizeof(float));
}

ccq_status check_sizes(int64_t n, int64_t rows, int width) {
    if (n < 0 || rows < 1 || width < 1)
        return op_fail(CCQ_ERR_INVALID_ARG, "bad sizes n=%lld rows=%lld width=%d", static_cast<long long>(n),
                       static_cast<long long>(rows), width);
    return CCQ_OK;
}

ccq_status check_grad_sizes(int64_t n, int64_t rows, int width) {
    ccq_status st = check_sizes(n, rows, width);
    if (st != CCQ_OK) return st;
    if (n > (1 << 30) || rows > (1 << 30))
        return op_fail(CCQ_ERR_UNSUPPORTED, "n=%lld rows=%lld: supported up to 2^30", static_cast<long long>(n),
                       static_cast<long long>(rows));
    return CCQ_OK;
}

ccq_status check_rows(const char *name, const void *p, ccq_dtype dtype, int64_t stride, int64_t rows, int width) {
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "%s: unknown dtype %d", name, dtype);
    if (rows > 1 && stride < width)
        return op_fail(CCQ_ERR_INVALID_ARG, "%s: row stride %lld is below the width %d", name,
                       static_cast<long long>(stride), width);
    return op_pointer(name, p, dtype_bytes(dtype));
}

ccq_status check_ids(const void *ids, int id_bytes) {
    if (id_bytes != 4 && id_bytes != 8) return op_fail(CCQ_ERR_INVALID_ARG, "id_bytes=%d: 4 or 8", id_bytes);
    return op_pointer("ids", ids, id_bytes);
}

}  // namespace
}  // namespace ccq

using namespace ccq;

extern "C" {

ccq_status ccq_embed(const void *table, ccq_dtype dtype, int64_t table_stride, const void *ids, int id_bytes, int64_t n,
                     int64_t rows, int width, float scale, void *out, int64_t out_stride, void *stream) {
    ccq_status st = check_sizes(n, rows, width);
    if (st != CCQ_OK) return st;
    if (n >= (static_cast<int64_t>(1) << 33))
        return op_fail(CCQ_ERR_UNSUPPORTED, "n=%lld: supported below 2^33", static_cast<long long>(n));
    if ((st = check_rows("table", table, dtype, table_stride, rows, width)) != CCQ_OK) return st;
    if (n == 0) return CCQ_OK;
    if ((st = check_ids(ids, id_bytes)) != CCQ_OK) return st;
    if ((st = check_rows("out", out, dtype, out_stride, n, width)) != CCQ_OK) return st;
    const int es = dtype_bytes(dtype);
    int b = access_bytes(static_cast<uintptr_t>(width) * es);
    b = row_access(table, table_stride, es, rows, b);
    b = row_access(out, out_stride, es, n, b);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto go = [&](auto fn) { return fn(table, table_stride, ids, id_bytes, n, rows, width, scale, out, out_stride, s); };
    cudaError_t e;
    if (dtype == CCQ_BF16)
        e = b == 16  ? go(launch_embed<__nv_bfloat16, 8>)
            : b == 8 ? go(launch_embed<__nv_bfloat16, 4>)
            : b == 4 ? go(launch_embed<__nv_bfloat16, 2>)
                     : go(launch_embed<__nv_bfloat16, 1>);
    else
        e = b == 16 ? go(launch_embed<float, 4>) : b == 8 ? go(launch_embed<float, 2>) : go(launch_embed<float, 1>);
    return op_cuda(e, "embedding lookup launch");
}

ccq_status ccq_embed_grad_workspace_size(int64_t n, int64_t rows, int width, size_t *bytes) {
    ccq_status st = check_grad_sizes(n, rows, width);
    if (st != CCQ_OK) return st;
    if (!bytes) return op_fail(CCQ_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = grad_workspace(n, rows, width);
    return CCQ_OK;
}

ccq_status ccq_embed_grad(const void *dout, ccq_dtype dtype, int64_t dout_stride, const void *ids, int id_bytes, int64_t n,
                          int64_t rows, int width, float scale, int64_t padding_id, void *dtable, ccq_dtype grad_dtype,
                          int64_t dtable_stride, void *workspace, size_t workspace_bytes, void *stream) {
    ccq_status st = check_grad_sizes(n, rows, width);
    if (st != CCQ_OK) return st;
    if ((st = check_rows("dtable", dtable, grad_dtype, dtable_stride, rows, width)) != CCQ_OK) return st;
    if (n > 0) {
        if ((st = check_ids(ids, id_bytes)) != CCQ_OK) return st;
        if ((st = check_rows("dout", dout, dtype, dout_stride, n, width)) != CCQ_OK) return st;
    }
    if (padding_id >= rows)
        return op_fail(CCQ_ERR_INVALID_ARG, "padding_id=%lld is outside the table of %lld rows",
                       static_cast<long long>(padding_id), static_cast<long long>(rows));
    const size_t need = grad_workspace(n, rows, width);
    if ((st = op_pointer("workspace", workspace, 16)) != CCQ_OK) return st;
    if (workspace_bytes < need)
        return op_fail(CCQ_ERR_INVALID_ARG, "workspace of %zu bytes, needs %zu", workspace_bytes, need);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const size_t list = round16(static_cast<size_t>(n) * 4);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    SortArgs so = {};
    so.ids = ids;
    so.id_bytes = id_bytes;
    so.n = static_cast<int>(n);
    so.rows = rows;
    so.padding = padding_id;
    const int bits = key_bits(rows);
    so.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    so.digit = (bits + so.passes - 1) / so.passes;
    for (int k = 0; k < 2; ++k) {
        so.key[k] = reinterpret_cast<uint32_t *>(ws + (2 * k) * list);
        so.pos[k] = reinterpret_cast<uint32_t *>(ws + (2 * k + 1) * list);
    }
    so.status = device_status_word();
    so.pieces = static_cast<int>(piece_count(n, rows));
    so.piece_start = reinterpret_cast<int *>(ws + 4 * list);
    const size_t starts = round16((static_cast<size_t>(so.pieces) + 1) * 4);
    so.joins = reinterpret_cast<int *>(ws + 4 * list + starts);
    const size_t smem = (kSortWarps + kSortCtas) * (static_cast<size_t>(1) << so.digit) * sizeof(uint32_t);
    cudaError_t e = allow_shared<embed_sort_kernel>((kSortWarps + kSortCtas) * (1 << kMaxDigit) * static_cast<int>(sizeof(uint32_t)));
    if (e != cudaSuccess) return op_cuda(e, "sort kernel attribute");
    embed_sort_kernel<<<kSortCtas, kSortThreads, smem, s>>>(so);
    if ((e = cudaGetLastError()) != cudaSuccess) return op_cuda(e, "sort launch");
    SumArgs a = {};
    a.dout = dout;
    a.dout_stride = dout_stride;
    a.key = so.key[(so.passes + 1) & 1];
    a.pos = so.pos[(so.passes + 1) & 1];
    a.n = so.n;
    a.rows = static_cast<int>(rows);
    a.width = width;
    a.scale = scale;
    a.dtable = dtable;
    a.dtable_stride = dtable_stride;
    a.piece_start = so.piece_start;
    a.joins = so.joins;
    a.part = reinterpret_cast<float *>(ws + 4 * list + 2 * starts);
    a.pieces = so.pieces;
    const int es = dtype_bytes(dtype), eo = dtype_bytes(grad_dtype);
    // elements an access may hold in both operands, at most 16 bytes of the wider type
    int b = row_access(dtable, dtable_stride, eo, rows, access_bytes(static_cast<uintptr_t>(width) * eo)) / eo;
    if (n > 0) b = std::min(b, row_access(dout, dout_stride, es, n, access_bytes(static_cast<uintptr_t>(width) * es)) / es);
    using B = __nv_bfloat16;
    if (dtype == CCQ_BF16 && grad_dtype == CCQ_BF16)
        e = b >= 8 ? launch_sum<B, B, 8>(a, s) : b >= 2 ? launch_sum<B, B, 2>(a, s) : launch_sum<B, B, 1>(a, s);
    else if (dtype == CCQ_BF16)
        e = b >= 4 ? launch_sum<B, float, 4>(a, s) : b >= 2 ? launch_sum<B, float, 2>(a, s) : launch_sum<B, float, 1>(a, s);
    else if (grad_dtype == CCQ_BF16)
        e = b >= 4 ? launch_sum<float, B, 4>(a, s) : b >= 2 ? launch_sum<float, B, 2>(a, s) : launch_sum<float, B, 1>(a, s);
    else
        e = b >= 4 ? launch_sum<float, float, 4>(a, s) : b >= 2 ? launch_sum<float, float, 2>(a, s)
                                                               : launch_sum<float, float, 1>(a, s);
    return op_cuda(e, "embedding gradient launch");
}

}  // extern "C"

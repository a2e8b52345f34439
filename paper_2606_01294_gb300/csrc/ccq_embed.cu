// ccq_embed.cu -- embedding lookup with scaling and the gradient of its table (ccq_ops.h).
//
// Lookup: out[i] = scale * table[ids[i]], a copy of n rows; bound by HBM (each row read once and
// written once).  32768 rows of 2048 bf16: 33 us, 8.1 TB/s of rows (frequent rows come from L2); 256 rows: 4.3 us, the
// launch.
//
// Gradient: dtable[r] = scale * sum of dout[i] over the i with ids[i] = r.  Each row of dout is read
// once and each row of dtable written once; no sum depends on the order of atomics:
//   1. embed_sort_kernel: one cluster of CTAs sorts (id, i) stably, all passes in one launch; the clusters beside it
//      write the rows that no id names (most of a vocabulary's), which hides the sort's latency.
//   2. embed_sum_kernel: the sorted entries are cut into pieces of kPiece, so that frequent ids cost no
//      more than others.  A warp takes a piece of a column slice, adds its entries and writes a row where its
//      run of equal ids ends.  A run that ends in the next piece is finished by the piece in which it begins; of
//      longer ones every piece leaves its part in the workspace.
//   3. embed_join_kernel: adds the parts of the runs over three pieces and more, in order.
// (Few ids need none of it: embed_few_kernel.)
// 16384 x 2048 bf16 into 32000 fp32 rows (329 MB, 48.6 us at the copy rate): 70 us, of which the zeros beside the sort are
// about 38 (213 MB, 5.6 TB/s; a plain fill of that size runs at 3.9), the sums 23 (116 MB, 5 TB/s), the join 6 and the
// gaps between launches the rest.  With short lists the sort's latency (16 to 30 us) is most of it.
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
    bool known[kLookupRows];
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
        const int64_t i = first + r * blockDim.y;
        id[r] = i < n ? load_index(ids, id_bytes, i) : 0;
        known[r] = id[r] >= 0 && id[r] < rows;
        if (!known[r]) {
            id[r] = 0;
            if (threadIdx.x == 0) note_index(status);
        }
    }
    constexpr int K = N * sizeof(T) <= 4 ? 4 : 1;  // columns at once: narrow accesses need more of them
    for (int c0 = threadIdx.x; c0 < packs; c0 += K * blockDim.x) {
        Pack<T, N> v[kLookupRows][K];
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                // (without conditions, so that all loads stay under way: past the end the last access, for an id outside row 0)
                const int c = min(c0 + k * static_cast<int>(blockDim.x), packs - 1);
                v[r][k] = load_plain<T, N>(table + id[r] * table_stride + static_cast<int64_t>(c) * N);
            }
        }
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
            const int64_t i = first + r * blockDim.y;
            if (i >= n) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = c0 + k * blockDim.x;
                if (c >= packs) continue;
                float f[N];
                unpack(v[r][k], f);
#pragma unroll
                for (int e = 0; e < N; ++e) f[e] = known[r] ? f[e] * scale : 0.f;
                pack(f, v[r][k]);
                store_stream<T, N>(out + i * out_stride + static_cast<int64_t>(c) * N, v[r][k]);
            }
        }
    }
}

template <typename T, int N>
cudaError_t launch_embed(const void *table, int64_t table_stride, const void *ids, int id_bytes, int64_t n,
                         int64_t rows, int width, float scale, void *out, int64_t out_stride, int *status, cudaStream_t s) {
    const int packs = width / N;
    int tx = 32;
    while (tx < kLookupThreads && tx < packs) tx *= 2;
    const int ty = kLookupThreads / tx;
    const unsigned grid = static_cast<unsigned>((n + ty * kLookupRows - 1) / (ty * kLookupRows));
    embed_kernel<T, N><<<grid, dim3(tx, ty), 0, s>>>(
        static_cast<const T *>(table), table_stride, ids, id_bytes, n, rows, packs, scale, static_cast<T *>(out),
        out_stride, status);
    return cudaGetLastError();
}

// ---------------------------------------------------------------- sort

constexpr int kMostCtas = 16;  // of the sort's cluster
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxDigit = 9;  // bits of a pass
constexpr int kHeld = 8;      // entries a lane keeps in registers; up to these, the passes exchange them in shared memory
constexpr int kPiece = 32;    // entries of a piece, one a lane

struct SortArgs {
    const void *ids;
    int id_bytes;
    int n;
    int64_t rows, padding;
    int passes, digit;
    uint2 *list[2];    // (key, position); the last pass writes list[(passes - 1) & 1], or list[0] where entries are held
    int *joins;  // their count, set to 0 (embed_sum_kernel)
    int *status;
    int ctas;  // of a cluster
    uint8_t *dtable;  // the CTAs behind the first cluster write its rows without entries
    int64_t row_bytes, row_stride;
    int access, present_words;  // bytes of a store, and words of a CTA's bitmap of its rows
};

// Entries of a warp, a multiple of 32.
__host__ __device__ inline int warp_entries(int n, int ctas) { return ((n + ctas * kSortWarps - 1) / (ctas * kSortWarps) + 31) & ~31; }
__host__ __device__ inline bool sort_holds(int n, int ctas) { return warp_entries(n, ctas) <= 32 * kHeld; }
constexpr int kSortMostShared = 204800;  // bytes
inline int sort_shared_words(int digit, int ctas) { return kSortWarps * ((1 << digit) + 1) + (ctas + 1) * (1 << digit); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_address(const void *p, int cta) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(cta));
    return a;
}
__device__ __forceinline__ void cluster_store(uint4 *p, int cta, uint4 v) {
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_address(p, cta)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}
__device__ __forceinline__ void cluster_store(uint2 *p, int cta, uint2 v) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(cluster_address(p, cta)), "r"(v.x), "r"(v.y) : "memory");
}
// Zeros to the rows that no id names: CTA `part` of `parts` looks after the rows r with r % parts = part.
__device__ __forceinline__ void zero_absent_rows(const SortArgs &a, uint32_t part, uint32_t parts, uint32_t *present) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t mine = a.rows > part ? (a.rows - part + parts - 1) / parts : 0;
    for (int w = tid; w < a.present_words; w += kSortThreads) present[w] = 0;
    __syncthreads();
    constexpr int kAtOnce = 8;
    for (int i0 = tid; i0 < a.n; i0 += kAtOnce * kSortThreads) {
        int64_t id[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int i = i0 + q * kSortThreads;
            id[q] = i >= a.n ? -1 : a.id_bytes == 8 ? static_cast<const int64_t *>(a.ids)[i] : static_cast<const int32_t *>(a.ids)[i];
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            if (id[q] < 0 || id[q] >= a.rows || id[q] == a.padding) continue;
            const uint32_t r = static_cast<uint32_t>(id[q]), at = r / parts;
            if (r - at * parts == part) atomicOr(&present[at >> 5], 1u << (at & 31));
        }
    }
    __syncthreads();
    for (int64_t q = warp; q < mine; q += kSortWarps) {
        if ((present[q >> 5] >> (q & 31)) & 1) continue;
        uint8_t *row = a.dtable + (q * parts + part) * a.row_stride;
        if (a.access == 16) {
            for (int64_t c = lane * 16; c < a.row_bytes; c += 512) __stcs(reinterpret_cast<uint4 *>(row + c), make_uint4(0, 0, 0, 0));
        } else if (a.access >= 4) {
            for (int64_t c = lane * 4; c < a.row_bytes; c += 128) __stcs(reinterpret_cast<uint32_t *>(row + c), 0u);
        } else {
            for (int64_t c = lane * 2; c < a.row_bytes; c += 64) __stcs(reinterpret_cast<uint16_t *>(row + c), static_cast<uint16_t>(0));
        }
    }
}

// Every warp owns a contiguous range of the entries, warps and CTAs in order, so ranks within a warp, sums over
// the warps before it and over the CTAs before that keep equal digits in order.  Invalid and padding ids get the
// key `rows`, behind every row.  All passes run in one launch.  Its time is latency: n = 16384 takes two passes of about
// five barriers each.  A lane finds the others with its digit by a ballot for each bit (match.any takes a time that grows with
// the number of different digits, 2000 cycles a step for 32 warps of random ones), and up to 8192 entries a CTA (131072 with
// 16) pass from CTA to CTA in shared memory (through global memory a pass took 6000 cycles for its stores and loads alone).
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint32_t smem[];
    const int ctas = a.ctas;
    if (static_cast<int>(blockIdx.x) >= ctas) {  // (whole clusters)
        zero_absent_rows(a, blockIdx.x - ctas, gridDim.x - ctas, smem);
        return;
    }
    const int bins = 1 << a.digit, row = bins + 1;  // (a column of counts spans all banks)
    uint32_t *counts = smem;                         // [kSortWarps][row]: a warp's entries, then those of the warps before it
    uint32_t *totals = counts + kSortWarps * row;    // [ctas][bins]: every CTA's entries (16-byte aligned: 32 rows)
    uint32_t *base = totals + ctas * bins;      // [bins]: this CTA's entries, then its first slot
    uint2 *xchg = reinterpret_cast<uint2 *>(smem + ((kSortWarps * row + (ctas + 1) * bins + 1) & ~1));  // this CTA's slots
    __shared__ uint32_t scan[kSortWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const int per = warp_entries(a.n, ctas), mine_slots = per * kSortWarps;
    const bool held = sort_holds(a.n, ctas);
    const int64_t lo64 = static_cast<int64_t>(cta * kSortWarps + warp) * per;
    const int lo = static_cast<int>(lo64 < a.n ? lo64 : a.n);
    const int hi = lo + (a.n - lo < per ? a.n - lo : per);
    uint32_t *mine = counts + warp * row;
    cluster_arrive();  // waited for before the first store to another CTA: all run by then
    if (cta == 0 && tid == 0) *a.joins = 0;
    auto key_from = [&](int64_t id) -> uint32_t {
        if (id < 0 || id >= a.rows) {
            note_index(a.status);
            return static_cast<uint32_t>(a.rows);
        }
        return static_cast<uint32_t>(id == a.padding ? a.rows : id);
    };
    uint2 kp[kHeld];
    uint32_t slot[kHeld];
    if (held) {
        int64_t id[kHeld];
        if (a.id_bytes == 8) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q) id[q] = lo + q * 32 + lane < hi ? static_cast<const int64_t *>(a.ids)[lo + q * 32 + lane] : 0;
        } else {
#pragma unroll
            for (int q = 0; q < kHeld; ++q) id[q] = lo + q * 32 + lane < hi ? static_cast<const int32_t *>(a.ids)[lo + q * 32 + lane] : 0;
        }
#pragma unroll
        for (int q = 0; q < kHeld; ++q) kp[q] = make_uint2(key_from(id[q]), static_cast<uint32_t>(lo + q * 32 + lane));
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit;
        const uint2 *from = a.list[(pass + 1) & 1];
        uint2 *to = a.list[pass & 1];
        auto entry = [&](int i) {
            return pass ? from[i] : make_uint2(key_from(load_index(a.ids, a.id_bytes, i)), static_cast<uint32_t>(i));
        };
        if (held && pass) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q)
                if (lo + q * 32 + lane < hi) kp[q] = xchg[warp * per + q * 32 + lane];
        }
        for (int i = tid; i < kSortWarps * row; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        // an entry's place among its warp's of the same digit
        auto place = [&](uint32_t key, bool live) -> uint32_t {
            const uint32_t d = (key >> shift) & (bins - 1);
            uint32_t same = __ballot_sync(~0u, live);
            for (int bit = 0; bit < a.digit; ++bit) {
                const bool set = (d >> bit) & 1;
                const uint32_t with = __ballot_sync(~0u, set);
                same &= set ? with : ~with;
            }
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
                if (lo + q * 32 < hi) slot[q] = place(kp[q].x, lo + q * 32 + lane < hi);
        } else {
            for (int i0 = lo; i0 < hi; i0 += 32) place(i0 + lane < hi ? entry(i0 + lane).x : 0, i0 + lane < hi);
        }
        __syncthreads();
        if (pass == 0) cluster_wait();
        // counts become those of the warps before; four lanes share a bin's 32 (their banks differ)
        for (int bin = tid >> 2; bin < bins; bin += kSortThreads / 4) {
            constexpr int kShare = kSortWarps / 4;
            uint32_t *from = counts + (tid & 3) * kShare * row + bin, c[kShare], sum = 0;
#pragma unroll
            for (int w = 0; w < kShare; ++w) c[w] = from[w * row];
#pragma unroll
            for (int w = 0; w < kShare; ++w) sum += c[w];
            uint32_t inc = sum;
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                const uint32_t t = __shfl_up_sync(0xfu << (lane & 28), inc, o, 4);
                if ((tid & 3) >= o) inc += t;
            }
            if ((tid & 3) == 3) base[bin] = inc;
            uint32_t at = inc - sum;
#pragma unroll
            for (int w = 0; w < kShare; ++w) {
                from[w * row] = at;
                at += c[w];
            }
        }
        __syncthreads();
        // this CTA's entries of every bin to all CTAs, four bins a store
        for (int q = tid; q < ctas * bins / 4; q += kSortThreads) {
            const int to = q / (bins / 4), quad = q - to * (bins / 4);
            cluster_store(reinterpret_cast<uint4 *>(&totals[cta * bins]) + quad, to, reinterpret_cast<const uint4 *>(base)[quad]);
        }
        cluster_arrive();
        cluster_wait();
        uint32_t all = 0, before = 0;
        if (tid < bins) {
#pragma unroll 4
            for (int c = 0; c < ctas; ++c) {
                const uint32_t t = totals[c * bins + tid];
                if (c < cta) before += t;
                all += t;
            }
        }
        // exclusive scan of `all` over the bins
        uint32_t inc = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 31) scan[warp] = inc;
        __syncthreads();
        if (tid < bins) {
            uint32_t b = inc - all + before;
            for (int w = 0; w < warp; ++w) b += scan[w];
            base[tid] = b;
        }
        __syncthreads();
        if (held) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                if (lo + q * 32 + lane >= hi) continue;
                const uint32_t d = (kp[q].x >> shift) & (bins - 1);
                const uint32_t at = slot[q] + mine[d] + base[d], owner = at / static_cast<uint32_t>(mine_slots);
                cluster_store(&xchg[at - owner * mine_slots], static_cast<int>(owner), kp[q]);
            }
        } else {
            // (place() counts on from the warps before this one)
            for (int i0 = lo; i0 < hi; i0 += 32) {
                const bool live = i0 + lane < hi;
                const uint2 e = live ? entry(i0 + lane) : make_uint2(0, 0);
                const uint32_t at = place(e.x, live) + base[(e.x >> shift) & (bins - 1)];
                if (live) to[at] = e;
            }
        }
        cluster_arrive();  // the next pass reads what the other CTAs wrote, and `totals` may be written again
        cluster_wait();
    }
    if (!held) return;
    // this CTA's slots
    const int first_slot = static_cast<int>(static_cast<int64_t>(cta) * mine_slots < a.n ? cta * mine_slots : a.n);
    const int slots = a.n - first_slot < mine_slots ? a.n - first_slot : mine_slots;
    for (int j = tid; j < slots; j += kSortThreads) a.list[0][first_slot + j] = xchg[j];
}

// ---------------------------------------------------------------- sums

struct SumArgs {
    const void *dout;
    int64_t dout_stride;
    const uint2 *list;  // sorted (key, position)
    int *count;   // of joins
    int2 *joins;  // (first, last piece) of the runs over three pieces and more
    int n, rows, width, packs;
    float scale;
    void *dtable;
    int64_t dtable_stride;
    float *part;  // [pieces][2][width]: what a piece holds of a run from before it, and of a run it leaves open
    int pieces;
};

constexpr int kSumThreads = 256;
constexpr int kJoinThreads = 256;

template <typename T, typename O, int N> __global__ void __launch_bounds__(kSumThreads, (N <= 2 ? 768 : 1024) / kSumThreads) embed_sum_kernel(SumArgs a) {
    constexpr int K = N <= 2 ? 4 : 1;        // accesses of a lane
    constexpr int kFlight = N >= 8 ? 4 : 8;  // entries whose loads are under way at once
    grid_wait();
    const int lane = threadIdx.x & 31;
    const int slices = (a.packs + 32 * K - 1) / (32 * K);
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kSumThreads / 32) + (threadIdx.x >> 5);
    const int64_t piece = warp / slices;
    if (piece >= a.pieces) return;
    const int slice = static_cast<int>(warp - piece * slices);
    const int c = slice * 32 * K + lane;
    const int live = c < a.packs ? (a.packs - c + 31) / 32 : 0;  // accesses of this lane within the row (K or more: all)
    // Loads are made without conditions, so that all stay under way: a lane past the row's end reads its last access, and what
    // is past the last entry the batch's first.
    const T *dout = static_cast<const T *>(a.dout);
    int offset[K];
#pragma unroll
    for (int j = 0; j < K; ++j) offset[j] = (c + 32 * j < a.packs ? c + 32 * j : a.packs - 1) * N;
    O *dtable = static_cast<O *>(a.dtable) + static_cast<int64_t>(c) * N;
    const int i0 = static_cast<int>(piece * kPiece);
    const uint32_t none = ~0u;
    // this piece's entries and those of the next, one a lane, and the keys of the entries before this piece, before the
    // one before it, and behind the next
    const uint2 e = i0 + lane < a.n ? a.list[i0 + lane] : make_uint2(none, 0);
    const uint2 e2 = i0 + kPiece + lane < a.n ? a.list[i0 + kPiece + lane] : make_uint2(none, 0);
    const uint32_t before0 = i0 > 0 ? a.list[i0 - 1].x : none, before1 = i0 > kPiece ? a.list[i0 - kPiece - 1].x : none;
    const uint32_t behind2 = i0 + 2 * kPiece < a.n ? a.list[i0 + 2 * kPiece].x : none;
    const uint32_t first = __shfl_sync(~0u, e.x, 0), last = __shfl_sync(~0u, e.x, kPiece - 1), next = __shfl_sync(~0u, e2.x, 0);
    // entries behind the last row's (invalid and padding ids) are left out
    const int own = __popc(__ballot_sync(~0u, e.x < static_cast<uint32_t>(a.rows)));
    if (!own) return;
    const uint32_t same = __ballot_sync(~0u, e.x == first);
    bool head = before0 == first;  // the first run has entries before this piece
    int skip = 0;
    // a run that began in the piece before and ends here is finished there
    if (head && before1 != first && !(same == ~0u && next == first)) {
        skip = __popc(same);
        head = false;
    }
    // the last run, if it goes on in the next piece: finished here, if it began here and ends there
    int more = 0;
    bool open = own == kPiece && next == last;
    if (open && skip < kPiece && !(head && same == ~0u)) {
        const uint32_t on = __ballot_sync(~0u, e2.x == last);
        if (!(on == ~0u && behind2 == last)) {
            more = __popc(on);
            open = false;
        }
    }
    if (skip == kPiece) open = false;
    float acc[K][N];
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int q = 0; q < N; ++q) acc[j][q] = 0.f;
    };
    auto leave = [&](int which) {  // the sums to the workspace
        float *to = a.part + (piece * 2 + which) * a.width + c * N;
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < live)
#pragma unroll
                for (int q = 0; q < N; ++q) to[j * 32 * N + q] = acc[j][q];
    };
    clear();
    auto end_run = [&](uint32_t row) {
        if (head) {
            leave(0);
        } else {
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (j >= live) continue;
                Pack<O, N> o;
                float f[N];
#pragma unroll
                for (int q = 0; q < N; ++q) f[q] = acc[j][q] * a.scale;
                pack(f, o);
                store_stream<O, N>(dtable + static_cast<int64_t>(row) * a.dtable_stride + j * 32 * N, o);
            }
        }
        if (head && slice == 0) {
            // for the join: the piece with the run's first entry; the warp tries 32 places at a time
            int lo = 0, hi = i0;
            while (lo < hi) {
                const int stride = (hi - lo + 31) / 32, at = lo + lane * stride;
                const uint32_t below = __ballot_sync(~0u, at < hi && a.list[at < hi ? at : hi - 1].x < row);
                if (!below) break;
                const int from = lo + (__popc(below) - 1) * stride;  // the last place whose key is below
                hi = from + stride < hi ? from + stride : hi;
                lo = from + 1;
            }
            if (lane == 0) a.joins[atomicAdd(a.count, 1)] = make_int2(lo / kPiece, static_cast<int>(piece));
        }
        head = false;
        clear();
    };
    const int count = own + more;
    if (skip >= count) return;
    uint32_t run = skip < own ? __shfl_sync(~0u, e.x, skip) : last;
    for (int q0 = skip; q0 < count; q0 += kFlight) {
        Pack<T, N> x[kFlight][K];
#pragma unroll
        for (int q = 0; q < kFlight; ++q) {
            const int at = q0 + q < count ? q0 + q : q0;
            const uint32_t row = at < own ? __shfl_sync(~0u, e.y, at & 31) : __shfl_sync(~0u, e2.y, (at - own) & 31);
            const T *from = dout + static_cast<int64_t>(row) * a.dout_stride;
#pragma unroll
            for (int j = 0; j < K; ++j) x[q][j] = load_stream<T, N>(from + offset[j]);
        }
#pragma unroll
        for (int q = 0; q < kFlight; ++q) {
            const int at = q0 + q;
            if (at >= count) break;
            const uint32_t k = at < own ? __shfl_sync(~0u, e.x, at & 31) : last;
            if (k != run) {
                end_run(run);
                run = k;
            }
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float f[N];
                unpack(x[q][j], f);
#pragma unroll
                for (int d = 0; d < N; ++d) acc[j][d] += f[d];
            }
        }
    }
    if (!open) end_run(run);
    else leave(1);
}

// The runs over three pieces and more: the parts of the pieces before the one that ends the run, then that one's.  A CTA takes
// 64 columns of a row, 16 threads 4 columns each, in 16 strided sums over the pieces that are then added in order.
constexpr int kJoinColumns = 64;
constexpr int kJoinCtas = 608;
template <typename O> __global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(SumArgs a) {
    __shared__ float sums[16][kJoinColumns + 1];
    grid_wait();
    const int count = *a.count, chunks = (a.width + kJoinColumns - 1) / kJoinColumns;
    const int column = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
    for (int64_t job = blockIdx.x; job < static_cast<int64_t>(count) * chunks; job += gridDim.x) {
        const int2 span = a.joins[job / chunks];
        const int piece = span.y, c0 = static_cast<int>(job % chunks) * kJoinColumns;
        const uint32_t row = a.list[static_cast<int64_t>(piece) * kPiece].x;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int64_t p = span.x + group; p <= piece; p += 16) {
            const float *from = a.part + (p * 2 + (p < piece)) * a.width + c0 + column;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (c0 + column + q < a.width) s[q] += from[q];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[group][column + q] = s[q];
        __syncthreads();
        if (threadIdx.x < kJoinColumns && c0 + static_cast<int>(threadIdx.x) < a.width) {
            float t = 0.f;
#pragma unroll
            for (int g = 0; g < 16; ++g) t += sums[g][threadIdx.x];
            static_cast<O *>(a.dtable)[static_cast<int64_t>(row) * a.dtable_stride + c0 + threadIdx.x] = from_f32<O>(t * a.scale);
        }
    }
}

template <typename T, typename O, int N> cudaError_t launch_sum(SumArgs a, cudaStream_t s) {
    a.packs = a.width / N;
    const int columns = N <= 2 ? 128 : 32;  // accesses of a warp
    const int64_t warps = static_cast<int64_t>(a.pieces) * ((a.packs + columns - 1) / columns);
    const int per = kSumThreads / 32;
    cudaError_t e = launch_after(embed_sum_kernel<T, O, N>, static_cast<unsigned>((warps + per - 1) / per), kSumThreads,
                                 0, s, a);
    if (e != cudaSuccess) return e;
    return launch_after(embed_join_kernel<O>, kJoinCtas, kJoinThreads, 0, s, a);
}

// ---------------------------------------------------------------- few ids

// Up to kFewIds ids need no sort: every warp holds them all, eight a lane, and for each row it writes asks by ballots which
// are equal to it, and adds their entries in ascending order.  One launch, bound by the table's rows that it writes: 30 x 2048
// into 300 rows 6.3 us (the sort and the sums took 17), 100 x 2048 into 30000 fp32 rows 41 us (45), 6.0 TB/s.  More ids than
// these are better sorted: a frequent id's entries are one warp's here.
constexpr int kFewIds = 256;
constexpr int kFewThreads = 256;

struct FewArgs {
    const void *ids;
    int id_bytes, n, rows, width, packs, parts;  // parts: warps that share a row
    int64_t padding;
    const void *dout;
    int64_t dout_stride, dtable_stride;
    void *dtable;
    float scale;
    int *status;
};

template <typename T, typename O, int N> __global__ void __launch_bounds__(kFewThreads) embed_few_kernel(FewArgs a) {
    constexpr int K = N >= 8 ? 2 : 4;                 // accesses of a lane at once
    constexpr int kFlight = N >= 4 ? 2 : 4;           // entries at once
    __shared__ uint8_t lists[kFewThreads / 32][kFewIds];
    uint8_t *list = lists[threadIdx.x >> 5];
    const int lane = threadIdx.x & 31;
    uint32_t id[kFewIds / 32];
#pragma unroll
    for (int j = 0; j < kFewIds / 32; ++j) {
        const int i = j * 32 + lane;
        id[j] = ~0u;
        if (i >= a.n) continue;
        const int64_t v = load_index(a.ids, a.id_bytes, i);
        if (v < 0 || v >= a.rows) {
            if (blockIdx.x == 0 && threadIdx.x < 32) note_index(a.status);
        } else if (v != a.padding) {
            id[j] = static_cast<uint32_t>(v);
        }
    }
    const uint32_t jobs = static_cast<uint32_t>(a.rows) * static_cast<uint32_t>(a.parts), warps = gridDim.x * (kFewThreads / 32);
    for (uint32_t job = blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5); job < jobs; job += warps) {
        const uint32_t row = job / a.parts, part = job - row * a.parts;
        // the row's entries, in ascending order
        int count = 0;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kFewIds / 32; ++j) {
            const bool mine = id[j] == row;
            const uint32_t hit = __ballot_sync(~0u, mine);
            if (mine) list[count + __popc(hit & ((1u << lane) - 1))] = static_cast<uint8_t>(j * 32 + lane);
            count += __popc(hit);
        }
        __syncwarp();
        O *out = static_cast<O *>(a.dtable) + static_cast<int64_t>(row) * a.dtable_stride;
        for (int c0 = part * 32 * K; c0 < a.packs; c0 += a.parts * 32 * K) {
            float acc[K][N];
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[k][e] = 0.f;
            for (int q0 = 0; q0 < count; q0 += kFlight) {
                Pack<T, N> x[kFlight][K];
#pragma unroll
                for (int q = 0; q < kFlight; ++q) {
                    const T *from = static_cast<const T *>(a.dout) + list[min(q0 + q, count - 1)] * a.dout_stride;
#pragma unroll
                    for (int k = 0; k < K; ++k) x[q][k] = load_stream<T, N>(from + static_cast<int64_t>(min(c0 + k * 32 + lane, a.packs - 1)) * N);
                }
#pragma unroll
                for (int q = 0; q < kFlight; ++q) {
                    if (q0 + q >= count) break;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        float f[N];
                        unpack(x[q][k], f);
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[k][e] += f[e];
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = c0 + k * 32 + lane;
                if (c >= a.packs) continue;
                float f[N];
                Pack<O, N> o;
#pragma unroll
                for (int e = 0; e < N; ++e) f[e] = acc[k][e] * a.scale;
                pack(f, o);
                store_stream<O, N>(out + static_cast<int64_t>(c) * N, o);
            }
        }
    }
}

template <typename T, typename O, int N> cudaError_t launch_few(FewArgs a, cudaStream_t s) {
    a.packs = a.width / N;
    a.parts = std::min(256, (a.packs + 127) / 128);  // (rows and parts: below 2^31 jobs)
    const int64_t jobs = static_cast<int64_t>(a.rows) * a.parts;
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((jobs + kFewThreads / 32 - 1) / (kFewThreads / 32), sm_count_now() * 8));
    embed_few_kernel<T, O, N><<<grid, kFewThreads, 0, s>>>(a);
    return cudaGetLastError();
}

// launch(packs of N elements of T and O) with the widest packs that `b` elements allow.
template <template <typename, typename, int> class Launch, typename A>
cudaError_t by_types(ccq_dtype dtype, ccq_dtype grad_dtype, int b, const A &a, cudaStream_t s) {
    using B = __nv_bfloat16;
    if (dtype == CCQ_BF16 && grad_dtype == CCQ_BF16)
        return b >= 8 ? Launch<B, B, 8>::go(a, s) : b >= 2 ? Launch<B, B, 2>::go(a, s) : Launch<B, B, 1>::go(a, s);
    if (dtype == CCQ_BF16)
        return b >= 4 ? Launch<B, float, 4>::go(a, s) : b >= 2 ? Launch<B, float, 2>::go(a, s) : Launch<B, float, 1>::go(a, s);
    if (grad_dtype == CCQ_BF16)
        return b >= 4 ? Launch<float, B, 4>::go(a, s) : b >= 2 ? Launch<float, B, 2>::go(a, s) : Launch<float, B, 1>::go(a, s);
    return b >= 4 ? Launch<float, float, 4>::go(a, s) : b >= 2 ? Launch<float, float, 2>::go(a, s) : Launch<float, float, 1>::go(a, s);
}
template <typename T, typename O, int N> struct Few {
    static cudaError_t go(const FewArgs &a, cudaStream_t s) { return launch_few<T, O, N>(a, s); }
};
template <typename T, typename O, int N> struct Sums {
    static cudaError_t go(const SumArgs &a, cudaStream_t s) { return launch_sum<T, O, N>(a, s); }
};

int key_bits(int64_t rows) {  // keys 0 .. rows
    int b = 1;
    while ((static_cast<int64_t>(1) << b) <= rows) ++b;
    return b;
}

// CTAs of the sort's cluster.  More make it faster (16384 ids: 21 us with 8, 16 with 16) and leave fewer SMs to write
// zeros beside it (140, 112, 96 with 4, 8, 16): few where the rows that surely have no entry are many, 16 (beyond the
// portable size) where ids are.  16384 x 2048 into 32000 rows: 70, 74, 80 us; 60000 x 64 into 100000: 82, 53, 47.
int sort_ctas(int64_t n, int64_t rows, size_t row_bytes) {
    if (n > 32768) return kMostCtas;
    return rows > n && static_cast<size_t>(rows - n) * row_bytes > (static_cast<size_t>(64) << 20) ? 4 : 8;
}

// The sort's launch with clusters of `ctas`; `clusters`: those resident at once, asked for once a device and size.
cudaError_t sort_config(int ctas, cudaLaunchConfig_t *cfg, cudaLaunchAttribute *at, int *clusters) {
    static std::atomic<int> known[64][kMostCtas + 1];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    *cfg = {};
    cfg->gridDim = dim3(ctas);
    cfg->blockDim = dim3(kSortThreads);
    cfg->dynamicSmemBytes = kSortMostShared;
    at->id = cudaLaunchAttributeClusterDimension;
    at->val.clusterDim.x = ctas;
    at->val.clusterDim.y = at->val.clusterDim.z = 1;
    cfg->attrs = at;
    cfg->numAttrs = 1;
    const bool keep = dev >= 0 && dev < 64;
    if (keep && (*clusters = known[dev][ctas].load(std::memory_order_relaxed)) > 0) return cudaSuccess;
    if ((e = allow_shared<embed_sort_kernel>(kSortMostShared)) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    if ((e = cudaOccupancyMaxActiveClusters(clusters, embed_sort_kernel, cfg)) != cudaSuccess) return e;
    *clusters = std::max(2, *clusters);
    if (keep) known[dev][ctas].store(*clusters, std::memory_order_relaxed);
    return cudaSuccess;
}

int64_t piece_count(int64_t n) { return (n + kPiece - 1) / kPiece; }

size_t round16(size_t x) { return (x + 15) & ~static_cast<size_t>(15); }

size_t grad_workspace(int64_t n, int width) {
    if (n <= kFewIds) return 0;
    const size_t pieces = static_cast<size_t>(piece_count(n));
    return 2 * round16(static_cast<size_t>(n) * 8) + 16 + round16(pieces * 8) + round16(pieces * 2 * width * sizeof(float));
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
    if (n > (1 << 30) || rows > (1 << 23))
        return op_fail(CCQ_ERR_UNSUPPORTED, "n=%lld rows=%lld: supported up to 2^30 and 2^23", static_cast<long long>(n),
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
    int *status = nullptr;
    if ((st = op_status_word(&status)) != CCQ_OK) return st;
    const int es = dtype_bytes(dtype);
    int b = access_bytes(static_cast<uintptr_t>(width) * es);
    b = row_access(table, table_stride, es, rows, b);
    b = row_access(out, out_stride, es, n, b);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto go = [&](auto fn) { return fn(table, table_stride, ids, id_bytes, n, rows, width, scale, out, out_stride, status, s); };
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
    *bytes = grad_workspace(n, width);
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
    const size_t need = grad_workspace(n, width);
    if (need && (st = op_pointer("workspace", workspace, 16)) != CCQ_OK) return st;
    if (workspace_bytes < need)
        return op_fail(CCQ_ERR_INVALID_ARG, "workspace of %zu bytes, needs %zu", workspace_bytes, need);
    int *status = nullptr;
    if ((st = op_status_word(&status)) != CCQ_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // elements an access may hold in both operands, at most 16 bytes of the wider type
    const int es = dtype_bytes(dtype), eo = dtype_bytes(grad_dtype);
    const int out_bytes = row_access(dtable, dtable_stride, eo, rows, access_bytes(static_cast<uintptr_t>(width) * eo));
    int b = out_bytes / eo;
    if (n > 0) b = std::min(b, row_access(dout, dout_stride, es, n, access_bytes(static_cast<uintptr_t>(width) * es)) / es);
    if (n <= kFewIds) {
        FewArgs f = {};
        f.ids = ids;
        f.id_bytes = id_bytes;
        f.n = static_cast<int>(n);
        f.rows = static_cast<int>(rows);
        f.width = width;
        f.padding = padding_id;
        f.dout = dout;
        f.dout_stride = dout_stride;
        f.dtable = dtable;
        f.dtable_stride = dtable_stride;
        f.scale = scale;
        f.status = status;
        return op_cuda(by_types<Few>(dtype, grad_dtype, b, f, s), "embedding gradient launch");
    }
    const size_t list = round16(static_cast<size_t>(n) * 8);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    SortArgs so = {};
    so.ids = ids;
    so.id_bytes = id_bytes;
    so.n = static_cast<int>(n);
    so.rows = rows;
    so.padding = padding_id;
    const int bits = key_bits(rows);
    so.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    so.digit = std::max(2, (bits + so.passes - 1) / so.passes);  // (bins are told four at a time)
    for (int k = 0; k < 2; ++k) so.list[k] = reinterpret_cast<uint2 *>(ws + k * list);
    so.joins = reinterpret_cast<int *>(ws + 2 * list);
    so.status = status;
    so.ctas = sort_ctas(n, rows, static_cast<size_t>(width) * eo);
    const bool held = sort_holds(so.n, so.ctas);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at;
    int clusters = 0;
    cudaError_t e = sort_config(so.ctas, &cfg, &at, &clusters);
    if (e != cudaSuccess) return op_cuda(e, "sort kernel configuration");
    const int parts = (clusters - 1) * so.ctas;
    so.dtable = static_cast<uint8_t *>(dtable);
    so.row_bytes = static_cast<int64_t>(width) * eo;
    so.row_stride = dtable_stride * eo;
    so.access = out_bytes;
    so.present_words = static_cast<int>((rows + static_cast<int64_t>(parts) * 32 - 1) / (static_cast<int64_t>(parts) * 32));
    const size_t slots = held ? static_cast<size_t>(warp_entries(so.n, so.ctas)) * kSortWarps : 0;
    cfg.gridDim = dim3(so.ctas + parts);
    cfg.dynamicSmemBytes = std::max(sort_shared_words(so.digit, so.ctas) * sizeof(uint32_t) + 8 + slots * sizeof(uint2),
                                    so.present_words * sizeof(uint32_t));
    cfg.stream = s;
    e = cudaLaunchKernelEx(&cfg, embed_sort_kernel, so);
    if (e != cudaSuccess) return op_cuda(e, "sort launch");
    SumArgs a = {};
    a.dout = dout;
    a.dout_stride = dout_stride;
    a.list = so.list[held ? 0 : (so.passes - 1) & 1];
    a.n = so.n;
    a.rows = static_cast<int>(rows);
    a.width = width;
    a.scale = scale;
    a.dtable = dtable;
    a.dtable_stride = dtable_stride;
    a.count = so.joins;
    a.joins = reinterpret_cast<int2 *>(ws + 2 * list + 16);
    a.pieces = static_cast<int>(piece_count(n));
    a.part = reinterpret_cast<float *>(ws + 2 * list + 16 + round16(static_cast<size_t>(a.pieces) * 8));
    e = by_types<Sums>(dtype, grad_dtype, b, a, s);
    return op_cuda(e, "embedding gradient launch");
}

}  // extern "C"

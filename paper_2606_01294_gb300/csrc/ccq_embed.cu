// ccq_embed.cu -- embedding lookup with scaling and the gradient of its table (ccq_ops.h).
//
// Lookup: out[i] = scale * table[ids[i]], a copy of n rows; bound by HBM (each row read once and
// written once).
//
// Gradient: dtable[r] = scale * sum of dout[i] over the i with ids[i] = r.  Each row of dout is read
// once and each row of dtable written once; no sum depends on the order of atomics:
//   1. embed_sort_kernel: a stable radix sort of (id, i), one cluster of 8 CTAs, all passes in one launch.
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
constexpr int kPiece = 32;     // path steps of a piece

struct SortArgs {
    const void *ids;
    int id_bytes;
    int n;
    int64_t rows, padding;
    int passes, digit;
    uint32_t *key[2];
    uint32_t *pos[2];
    int *status;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ uint32_t cluster_load(const uint32_t *p, int cta) {
    uint32_t a, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(cta));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// Every warp owns a contiguous range of the entries, warps and CTAs in order, so ranks within a warp, sums over
// the warps before it and over the CTAs before that keep equal digits in order.  Invalid and padding ids get the
// key `rows`, behind every row.
__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) embed_sort_kernel(SortArgs a) {
    extern __shared__ uint32_t smem[];
    const int bins = 1 << a.digit;
    uint32_t *counts = smem;                   // [kSortWarps][bins], then the warp's next slot of each bin
    uint32_t *total = smem + kSortWarps * bins;  // [bins] entries of this CTA
    __shared__ uint32_t scan[kSortWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const int per = ((a.n + kSortCtas * kSortWarps - 1) / (kSortCtas * kSortWarps) + 31) & ~31;
    const int64_t lo64 = static_cast<int64_t>(cta * kSortWarps + warp) * per;
    const int lo = static_cast<int>(lo64 < a.n ? lo64 : a.n);
    const int hi = lo + (a.n - lo < per ? a.n - lo : per);
    uint32_t *mine = counts + warp * bins;
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit;
        const uint32_t *key = a.key[(pass + 1) & 1], *pos = a.pos[(pass + 1) & 1];
        uint32_t *key_out = a.key[pass & 1], *pos_out = a.pos[pass & 1];
        for (int i = tid; i < kSortWarps * bins; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        auto key_of = [&](int i) -> uint32_t {
            if (pass) return key[i];
            const int64_t id = load_index(a.ids, a.id_bytes, i);
            if (id < 0 || id >= a.rows) {
                note_index(a.status);
                return static_cast<uint32_t>(a.rows);
            }
            return static_cast<uint32_t>(id == a.padding ? a.rows : id);
        };
        for (int i = lo + lane; i < hi; i += 32) atomicAdd(&mine[(key_of(i) >> shift) & (bins - 1)], 1u);
        __syncthreads();
        // this CTA's entries of every bin, and the slot of each warp's first one among them
        uint32_t sum = 0;
        if (tid < bins) {
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = counts[w * bins + tid];
                counts[w * bins + tid] = sum;
                sum += c;
            }
            total[tid] = sum;
        }
        cluster_sync();
        uint32_t all = 0, before = 0;
        if (tid < bins)
            for (int c = 0; c < kSortCtas; ++c) {
                const uint32_t t = cluster_load(&total[tid], c);
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
        if (warp == 0) {
            uint32_t t = scan[lane];
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(~0u, t, o);
                if (lane >= o) t += u;
            }
            scan[lane] = t;
        }
        __syncthreads();
        if (tid < bins) {
            const uint32_t base = inc - all + (warp ? scan[warp - 1] : 0) + before;
            for (int w = 0; w < kSortWarps; ++w) counts[w * bins + tid] += base;
        }
        __syncthreads();
        for (int i0 = lo; i0 < hi; i0 += 32) {
            const int i = i0 + lane;
            const bool live = i < hi;
            const uint32_t k = live ? key_of(i) : 0;
            const uint32_t p = !live ? 0 : pass ? pos[i] : static_cast<uint32_t>(i);
            const uint32_t d = live ? (k >> shift) & (bins - 1) : ~0u;
            const uint32_t same = __match_any_sync(~0u, d);
            const int rank = __popc(same & ((1u << lane) - 1));
            uint32_t slot = 0;
            if (live) slot = mine[d] + rank;
            __syncwarp();
            if (live && rank == 0) mine[d] += __popc(same);
            __syncwarp();
            if (live) {
                key_out[slot] = k;
                pos_out[slot] = p;
            }
        }
        cluster_sync();  // the next pass reads what the other CTAs wrote, and `total` may be written again
    }
}

// ---------------------------------------------------------------- sums

struct SumArgs {
    const void *dout;
    int64_t dout_stride;
    const uint32_t *key, *pos;  // sorted entries
    int n, rows, width, packs;
    float scale;
    void *dtable;
    int64_t dtable_stride;
    float *part;  // [pieces][2][width]: what a piece holds of a row from before it, and of a row it leaves open
    int pieces;
};

// Entries with a key below v.
__device__ __forceinline__ int lower_bound(const uint32_t *key, int n, uint32_t v) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (key[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Entries among the first `step` steps of the path: entry i comes before the end of row key[i], so it is step
// i + key[i].
__device__ __forceinline__ int path_entries(const uint32_t *key, int n, int64_t step) {
    int lo = 0, hi = static_cast<int>(step < n ? step : n);
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (static_cast<int64_t>(mid) + key[mid] < step) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

constexpr int kSumThreads = 256;

template <typename T, typename O, int N> __global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(SumArgs a) {
    grid_wait();
    const int lane = threadIdx.x & 31;
    const int slices = (a.packs + 31) / 32;
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kSumThreads / 32) + (threadIdx.x >> 5);
    const int64_t piece = warp / slices;
    if (piece >= a.pieces) return;
    const int c = static_cast<int>(warp % slices) * 32 + lane;
    const bool live = c < a.packs;
    const T *dout = static_cast<const T *>(a.dout) + static_cast<int64_t>(c) * N;
    O *dtable = static_cast<O *>(a.dtable) + static_cast<int64_t>(c) * N;
    const int64_t step0 = piece * kPiece, step1 = step0 + kPiece;
    int i = path_entries(a.key, a.n, step0);
    const int i1 = path_entries(a.key, a.n, step1);
    int v = static_cast<int>(step0 - i);
    const int v1 = static_cast<int>(step1 - i1 < a.rows ? step1 - i1 : a.rows);
    const bool open = i > 0 && v < a.rows && a.key[i - 1] == static_cast<uint32_t>(v);
    bool head = open;  // the sum in hand belongs to a row with entries before this piece
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    for (;;) {
        // the entries of row v (none when it has no more in this piece)
        while (i < i1 && v < a.rows && a.key[i] == static_cast<uint32_t>(v)) {
            if (live) {
                float f[N];
                unpack(load_stream<T, N>(dout + static_cast<int64_t>(a.pos[i]) * a.dout_stride), f);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += f[e];
            }
            ++i;
        }
        if (v >= v1) break;
        if (live) {
            if (head) {
#pragma unroll
                for (int e = 0; e < N; ++e) a.part[piece * 2 * a.width + c * N + e] = acc[e];
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
    }
    if (live && v < a.rows) {
#pragma unroll
        for (int e = 0; e < N; ++e) a.part[(piece * 2 + 1) * a.width + c * N + e] = acc[e];
    }
}

// A CTA for each piece; it acts where the piece ends a row that began in an earlier one.
template <typename O> __global__ void __launch_bounds__(kSumThreads) embed_join_kernel(SumArgs a) {
    grid_wait();
    const int64_t piece = blockIdx.x;
    const int64_t step0 = piece * kPiece;
    const int i = path_entries(a.key, a.n, step0);
    const int v = static_cast<int>(step0 - i);
    if (i == 0 || v >= a.rows || a.key[i - 1] != static_cast<uint32_t>(v)) return;
    const int end = lower_bound(a.key, a.n, static_cast<uint32_t>(v) + 1);
    if (static_cast<int64_t>(end) + v >= step0 + kPiece) return;  // ends in a later piece
    const int64_t first = (static_cast<int64_t>(lower_bound(a.key, a.n, static_cast<uint32_t>(v))) + v) / kPiece;
    for (int c = threadIdx.x; c < a.width; c += kSumThreads) {
        float sum = 0.f;
        for (int64_t p = first; p < piece; ++p) sum += a.part[(p * 2 + 1) * a.width + c];
        sum += a.part[piece * 2 * a.width + c];
        static_cast<O *>(a.dtable)[static_cast<int64_t>(v) * a.dtable_stride + c] = from_f32<O>(sum * a.scale);
    }
}

template <typename T, typename O, int N> cudaError_t launch_sum(SumArgs a, cudaStream_t s) {
    a.packs = a.width / N;
    const int64_t warps = static_cast<int64_t>(a.pieces) * ((a.packs + 31) / 32);
    const int per = kSumThreads / 32;
    cudaError_t e = launch_after(embed_sum_kernel<T, O, N>, static_cast<unsigned>((warps + per - 1) / per), kSumThreads,
                                 0, s, a);
    if (e != cudaSuccess) return e;
    return launch_after(embed_join_kernel<O>, static_cast<unsigned>(a.pieces), kSumThreads, 0, s, a);
}

int key_bits(int64_t rows) {  // keys 0 .. rows
    int b = 1;
    while ((static_cast<int64_t>(1) << b) <= rows) ++b;
    return b;
}

int64_t piece_count(int64_t n, int64_t rows) { return (n + rows + kPiece - 1) / kPiece; }

size_t round16(size_t x) { return (x + 15) & ~static_cast<size_t>(15); }

size_t grad_workspace(int64_t n, int64_t rows, int width) {
    return 4 * round16(static_cast<size_t>(n) * 4) +
           round16(static_cast<size_t>(piece_count(n, rows)) * 2 * width * sizeof(float));
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
    const size_t smem = (kSortWarps + 1) * (static_cast<size_t>(1) << so.digit) * sizeof(uint32_t);
    cudaError_t e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (kSortWarps + 1) * (1 << kMaxDigit) * static_cast<int>(sizeof(uint32_t)));
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
    a.part = reinterpret_cast<float *>(ws + 4 * list);
    a.pieces = static_cast<int>(piece_count(n, rows));
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

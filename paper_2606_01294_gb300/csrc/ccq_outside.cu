// ccq_outside.cu -- zeros to the tokens of a packed batch that no sequence holds (ccq_ops.h).
//
// Row t is held where cu[s] <= t < cu[s + 1] for some s, the offsets held to 0 .. T as decay_span() does.  Offsets may go back, so
// that is asked of all of them: a CTA marks its rows in a bitmap, by all sequences, and writes the rows that stay unmarked.
// Words of 32 rows go round the CTAs, so that padding behind the last sequence, one run of rows, is written by all of them.
// Bound by its launch, 2 us, where little is left over (64 x 1000 tokens); 3000 sequences of 20 8 us, reading the offsets; 8000 rows of
// padding in 16 heads of 128 in bf16 9 us.
#include <algorithm>

#include "ccq_decay.cuh"

namespace ccq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWords = 2048;  // of a CTA at once: 8 KB, 65536 rows

// Marks words j, j + by, .. (to `last`) of a CTA's, which lie at base + j step, of those that rows begin .. end - 1 lie in.
__device__ __forceinline__ void mark(uint32_t *held, int begin, int end, int j, int last, int by, int base, int step) {
    const int w0 = begin / 32, w1 = (end - 1) / 32;
    for (; j <= last; j += by) {
        const int w = base + j * step;
        const uint32_t above = w == w0 ? 0xffffffffu << (begin % 32) : 0xffffffffu,
                       below = w == w1 ? 0xffffffffu >> (31 - (end - 1) % 32) : 0xffffffffu;
        atomicOr(&held[j], above & below);
    }
}

__global__ void __launch_bounds__(kThreads) outside_kernel(const OutsideArgs a) {
    __shared__ uint32_t held[kWords];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int T = static_cast<int>(a.T), step = gridDim.x, total = (T - 1) / 32 + 1;  // words
    for (int64_t base64 = blockIdx.x; base64 < total; base64 += static_cast<int64_t>(step) * kWords) {
        const int base = static_cast<int>(base64), words = min(kWords, (total - 1 - base) / step + 1);
        for (int j = tid; j < words; j += kThreads) held[j] = 0;
        __syncthreads();
        // a thread a sequence; one of more than two of the CTA's words is marked by its warp
#pragma unroll 4
        for (int64_t s0 = 0; s0 < a.sequences; s0 += kThreads) {
            const int64_t s = s0 + tid;
            int begin = 0, end = 0, j = 0, last = -1;
            if (s < a.sequences) {
                const int64_t from = load_index(a.cu, a.cu_bytes, s), to = load_index(a.cu, a.cu_bytes, s + 1);
                begin = static_cast<int>(min(max(from, static_cast<int64_t>(0)), a.T));
                end = static_cast<int>(min(max(to, static_cast<int64_t>(begin)), a.T));
                if (begin < end && (end - 1) / 32 >= base) {
                    j = begin / 32 > base ? (begin / 32 - base - 1) / step + 1 : 0;
                    last = min(words - 1, ((end - 1) / 32 - base) / step);
                }
            }
            const bool wide = last - j > 1;
            if (!wide) mark(held, begin, end, j, last, 1, base, step);
            for (uint32_t left = __ballot_sync(0xffffffffu, wide); left; left &= left - 1) {
                const int from = __ffs(left) - 1;
                mark(held, __shfl_sync(0xffffffffu, begin, from), __shfl_sync(0xffffffffu, end, from),
                     __shfl_sync(0xffffffffu, j, from) + lane, __shfl_sync(0xffffffffu, last, from), 32, base, step);
            }
        }
        __syncthreads();
        for (int j = 0; j < words; ++j) {
            const uint32_t rows = ~held[j];
            if (!rows) continue;
            for (int r = warp; r < 32; r += kWarps) {
                const int64_t t = 32 * (static_cast<int64_t>(base) + static_cast<int64_t>(j) * step) + r;
                if (!(rows >> r & 1) || t >= T) continue;
                for (int i = 0; i < a.count; ++i) {
                    const OutsideTensor &x = a.x[i];
                    uint8_t *row = static_cast<uint8_t *>(x.p) + t * x.token;
                    const int per_head = x.wide ? x.bytes / 16 : x.bytes / 2;
                    for (int k = lane; k < x.heads * per_head; k += 32) {
                        const int h = k / per_head, c = k % per_head;
                        if (x.wide)
                            *reinterpret_cast<uint4 *>(row + h * x.head + 16 * c) = make_uint4(0, 0, 0, 0);
                        else
                            *reinterpret_cast<uint16_t *>(row + h * x.head + 2 * c) = 0;
                    }
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace

OutsideTensor outside_tensor(void *p, int elem, int64_t token, int64_t head, int heads, int width) {
    OutsideTensor x = {p, token * elem, heads > 1 ? head * elem : 0, heads, width * elem, 0};
    x.wide = (reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(x.token) | static_cast<uintptr_t>(x.head) |
              static_cast<uintptr_t>(x.bytes)) % 16 == 0;
    return x;
}

cudaError_t launch_outside(const OutsideArgs &a, cudaStream_t s) {
    const int64_t words = (a.T + 31) / 32;
    if (!words || !a.count) return cudaSuccess;
    outside_kernel<<<static_cast<unsigned>(std::min<int64_t>(words, 2 * sm_count_now())), kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace ccq

using namespace ccq;

extern "C" {

ccq_status ccq_zero_outside(const ccq_heads *x, ccq_dtype dtype, int64_t T, int width, const void *cu, int cu_bytes,
                            int64_t num_seqs, void *stream) {
    if (!x) return op_fail(CCQ_ERR_INVALID_ARG, "x is NULL");
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", static_cast<int>(dtype));
    ccq_status st = check_tokens(1, T);
    if (st != CCQ_OK) return st;
    if (width < 1 || width > 65536) return op_fail(CCQ_ERR_INVALID_ARG, "head width %d: 1 to 65536", width);
    if (num_seqs < 0 || num_seqs > (1 << 24))
        return op_fail(CCQ_ERR_UNSUPPORTED, "%lld sequences: at most 2^24", static_cast<long long>(num_seqs));
    if (cu_bytes != 4 && cu_bytes != 8) return op_fail(CCQ_ERR_INVALID_ARG, "cu_bytes=%d: 4 or 8", cu_bytes);
    if ((st = op_pointer("cu", cu, cu_bytes)) != CCQ_OK) return st;
    if ((st = check_heads("x", *x, dtype, 1, T, width, true)) != CCQ_OK) return st;
    if (x->heads * width > (1 << 24)) return op_fail(CCQ_ERR_UNSUPPORTED, "at most 2^24 channels a token");
    if (T == 0) return CCQ_OK;
    OutsideArgs a = {};
    a.x[a.count++] = outside_tensor(x->p, dtype_bytes(dtype), x->token, x->head, static_cast<int>(x->heads), width);
    a.T = T;
    a.cu = cu;
    a.cu_bytes = cu_bytes;
    a.sequences = num_seqs;
    return op_cuda(launch_outside(a, static_cast<cudaStream_t>(stream)), "rows outside launch");
}

}  // extern "C"

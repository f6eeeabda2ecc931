// scd_clip.hip -- the norm of many tensors together, and their clipping by it (gfx950).
//
// n = sqrt(sum g^2), f = max / n if n > max else 1, out = f g.  Bound by memory: every element is read for the norm
// and read and written for the product.  The tensors' addresses and lengths travel in the launch's arguments
// (up to kSpans a launch), so that a call copies nothing to the GPU; a tensor is cut into chunks, and each
// workgroup takes a run of consecutive chunks.  Squares are summed in 64 bits: the square of a 32-bit value
// overflows 32 bits, and the 64-bit units are idle otherwise.  Each workgroup of the first kernel writes its sum; every
// workgroup of the second adds them all in the same order (a few KB from the cache) and scales its share.
#include <algorithm>
#include <cmath>

#include "scd_device.h"
#include "scd_feat.h"

namespace scd {
namespace feat {
namespace {

constexpr int kClipThreads = 256;
constexpr int kSpans = 100;         // per launch: the arguments stay below 4 KB
constexpr int kClipBlocks = 1024;   // workgroups of a launch at most
constexpr int kMaxSums = 8192;      // workgroups' sums in the workspace
constexpr int64_t kChunk = 8192;    // elements: 32 a thread
constexpr int64_t kMaxElements = int64_t(1) << 44;  // of a call: chunk numbers stay below 2^32

struct Span {
    const void* src;
    void* dst;
    int64_t n;
    uint32_t first;  // number of chunks before this span's
    uint8_t st, dt;
    uint16_t pad_;
};
struct Spans {
    Span s[kSpans];
    uint32_t count;
    uint32_t chunks;
};

// The span that holds a chunk.
__device__ __forceinline__ uint32_t span_of(const Spans& a, uint32_t chunk) {
    uint32_t lo = 0, hi = a.count;  // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.s[mid].first <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// The workgroup's sum of a value per thread, in thread order of a fixed tree; valid in thread 0.
__device__ __forceinline__ double block_sum(double x, double* lds) {
    x = group_sum_f64<64>(x);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    double s = 0.0;
    for (uint32_t w = 0; w < blockDim.x / 64; ++w) s += lds[w];
    __syncthreads();
    return s;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* __restrict__ p, int64_t n) {
    constexpr int V = 16 / sizeof(T), U = kChunk / (kClipThreads * V);
    double s = 0.0;
    if (n == kChunk) {
        Raw<V, T> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_raw<V>(p + (u * kClipThreads + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double x = (double)(float)r[u].t[i];
                s += x * x;
            }
    } else {
        for (int64_t i = threadIdx.x; i < n; i += kClipThreads) {
            const double x = (double)(float)p[i];
            s += x * x;
        }
    }
    return s;
}

template <typename S, typename D>
__device__ __forceinline__ void chunk_scale(const S* p, D* q, int64_t n, float f, float f2) {
    constexpr int V = 16 / (sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D)), U = kChunk / (kClipThreads * V);
    if (n == kChunk) {
        constexpr int B = U < 8 ? U : 8;
#pragma unroll
        for (int b = 0; b < U; b += B) {
            Raw<V, S> r[B];
#pragma unroll
            for (int u = 0; u < B; ++u) r[u] = load_raw<V>(p + ((b + u) * kClipThreads + threadIdx.x) * V);
#pragma unroll
            for (int u = 0; u < B; ++u) {
                float x[V];
                widen(r[u], x);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = x[i] * f2 * f;
                store_vec(q + ((b + u) * kClipThreads + threadIdx.x) * V, x);
            }
        }
    } else {
        for (int64_t i = threadIdx.x; i < n; i += kClipThreads) q[i] = (D)((float)p[i] * f2 * f);
    }
}

__global__ void __launch_bounds__(kClipThreads) k_clip_squares(Spans a, double* __restrict__ sums) {
    __shared__ double lds[kClipThreads / 64];
    const uint32_t c0 = (uint32_t)((uint64_t)a.chunks * blockIdx.x / gridDim.x);
    const uint32_t c1 = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / gridDim.x);
    double s = 0.0;
    uint32_t k = span_of(a, c0);
    for (uint32_t c = c0; c < c1; ++c) {
        while (k + 1 < a.count && a.s[k + 1].first <= c) ++k;
        const int64_t at = (int64_t)(c - a.s[k].first) * kChunk, n = min(kChunk, a.s[k].n - at);
        const void* const p = a.s[k].src;
        if (a.s[k].st == SCD_F32)
            s += chunk_squares((const float*)p + at, n);
        else if (a.s[k].st == SCD_BF16)
            s += chunk_squares((const bf16*)p + at, n);
        else
            s += chunk_squares((const f16*)p + at, n);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kClipThreads) k_clip_scale(Spans a, const double* __restrict__ sums, uint32_t n_sums,
                                                             float max_norm, float* __restrict__ norm_out) {
    __shared__ double lds[kClipThreads / 64];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < n_sums; i += kClipThreads) s += sums[i];
    const double norm = sqrt(block_sum(s, lds));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    // The factor is f f2: f2 is a power of two below 1 where the factor is too small for 32 bits' normal range.
    const double factor = norm <= (double)max_norm ? 1.0 : (double)max_norm / norm;  // NaN: NaN
    const float f2 = factor < 0x1p-100 ? 0x1p-64f : 1.0f, f = (float)(factor / (double)f2);
    const uint32_t c0 = (uint32_t)((uint64_t)a.chunks * blockIdx.x / gridDim.x);
    const uint32_t c1 = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / gridDim.x);
    if (c0 == c1) return;
    uint32_t k = span_of(a, c0);
    for (uint32_t c = c0; c < c1; ++c) {
        while (k + 1 < a.count && a.s[k + 1].first <= c) ++k;
        const Span& t = a.s[k];
        if (!t.dst || (t.dst == t.src && factor == 1.0)) continue;
        const int64_t at = (int64_t)(c - t.first) * kChunk, n = min(kChunk, t.n - at);
        if (t.st == SCD_F32)
            chunk_scale((const float*)t.src + at, (float*)t.dst + at, n, f, f2);
        else if (t.st == SCD_BF16 && t.dt == SCD_BF16)
            chunk_scale((const bf16*)t.src + at, (bf16*)t.dst + at, n, f, f2);
        else if (t.st == SCD_BF16)
            chunk_scale((const bf16*)t.src + at, (float*)t.dst + at, n, f, f2);
        else if (t.dt == SCD_F16)
            chunk_scale((const f16*)t.src + at, (f16*)t.dst + at, n, f, f2);
        else
            chunk_scale((const f16*)t.src + at, (float*)t.dst + at, n, f, f2);
    }
}

}  // namespace
}  // namespace feat
}  // namespace scd

using namespace scd::feat;

extern "C" int scd_clip_grads_workspace(int64_t* bytes) {
    if (!bytes) return fail(SCD_ERR_INVALID, "bytes is null");
    *bytes = kMaxSums * sizeof(double);
    return SCD_OK;
}

extern "C" int scd_clip_grads(const scd_span_t* spans, int64_t count, float max_norm, float* norm, void* workspace,
                              int64_t workspace_bytes, void* stream) {
    if (count < 0 || (count > 0 && !spans)) return fail(SCD_ERR_INVALID, "bad spans");
    if (!(max_norm >= 0.0f)) return fail(SCD_ERR_INVALID, "max_norm must be >= 0");
    if (!norm) return fail(SCD_ERR_INVALID, "null device pointer");
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < (int64_t)(kMaxSums * sizeof(double)))
        return fail(SCD_ERR_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)(kMaxSums * sizeof(double)));
    int64_t used = 0, total = 0;
    for (int64_t i = 0; i < count; ++i) {
        const scd_span_t& t = spans[i];
        if (!type_bytes(t.src_type) || (t.dst_type != t.src_type && t.dst_type != SCD_F32))
            return fail(SCD_ERR_UNSUPPORTED, "span %lld: float32, bfloat16 or float16 into that type or float32", (long long)i);
        if (t.n < 0 || t.n > kMaxElements - total || (t.n > 0 && !t.src)) return fail(SCD_ERR_INVALID, "span %lld: bad size or null pointer", (long long)i);
        if (t.n > 0 && t.dst == t.src && t.dst_type != t.src_type) return fail(SCD_ERR_INVALID, "span %lld: in place the types must be the same", (long long)i);
        used += t.n > 0;
        total += t.n;
    }
    const int64_t launches = std::max<int64_t>(1, ceil_div(used, kSpans));
    if (launches > kMaxSums) return fail(SCD_ERR_UNSUPPORTED, "more than %lld spans", (long long)kMaxSums * kSpans);
    // Workgroups' sums: every launch gets the same share of the workspace.
    const int64_t most = std::min<int64_t>(kClipBlocks, kMaxSums / launches);
    hipStream_t s = (hipStream_t)stream;
    double* const sums = (double*)workspace;
    uint32_t n_sums = 0;
    // The same groups of spans twice: for the sums, then for the product.
    for (int pass = 0; pass < 2; ++pass) {
        Spans a;
        a.count = 0;
        a.chunks = 0;
        bool first = true;
        const auto launch = [&] {
            if (pass == 0) {
                if (a.chunks == 0) return;
                const uint32_t blocks = (uint32_t)std::min<int64_t>(most, a.chunks);
                k_clip_squares<<<blocks, kClipThreads, 0, s>>>(a, sums + n_sums);
                n_sums += blocks;
            } else {
                const uint32_t blocks = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(2 * kClipBlocks, a.chunks));
                k_clip_scale<<<blocks, kClipThreads, 0, s>>>(a, sums, n_sums, max_norm, first ? norm : nullptr);
                first = false;
            }
            a.count = 0;
            a.chunks = 0;
        };
        for (int64_t i = 0; i < count; ++i) {
            const scd_span_t& t = spans[i];
            if (t.n == 0) continue;
            const int64_t chunks = ceil_div(t.n, kChunk);
            if (a.count == kSpans) launch();
            a.s[a.count++] = Span{t.src, t.dst, t.n, a.chunks, (uint8_t)t.src_type, (uint8_t)t.dst_type, 0};
            a.chunks += (uint32_t)chunks;
        }
        if (a.count || (pass == 1 && first)) launch();
    }
    return launched("scd_clip_grads");
}

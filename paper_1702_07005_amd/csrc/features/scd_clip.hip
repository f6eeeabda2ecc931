// scd_clip.hip -- the norm of many tensors together, and their clipping by it (gfx950).
//
// n = sqrt(sum g^2), f = max / n if n > max else 1, out = f g.  Bound by memory: every element is read for the norm
// and read and written for the product.  The tensors' addresses and lengths travel in the launch's arguments
// (up to kSpans a launch), so that a call copies nothing to the GPU; a tensor is cut into chunks, and each
// workgroup takes a run of consecutive chunks.  Squares are summed in 64 bits: the square of a 32-bit value
// overflows 32 bits, and the 64-bit units are idle otherwise.  Each workgroup of the first kernel writes its sum; every
// workgroup of the second adds them all in the same order (a few KB from the cache) and scales its share.
//
// Measured: 354 M weights from bf16 to fp32 490 us (2.1 GB that it cannot do without: 4.3 TB/s; with what is read twice
// and not from the cache, 5.4); 11 tensors of 160,000 weights in all 9.9 us, two launches.
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
// What the first kernel reads last and the second finds in the 256 MB cache; the rest is read past the caches, as are the
// results written.  350 M bf16 elements into fp32: 560 us through the caches, 489 so.
// On both sides of the limit: 700 MB of bf16 into fp32 516 us with 160 MB kept, 511 with 192, 508 with 224, 505 with 256, 513
// with all of it; 300 MB of fp32 into as many 159, 154, 150, 147 and 151.
constexpr int64_t kKeepBytes = int64_t(224) << 20;
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
    uint32_t chunk;  // elements of a chunk
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

// f(column, whole) for this thread's vectors of V of n elements; the last one may hold fewer.
template <int V, typename F>
__device__ __forceinline__ void for_vectors(int64_t n, F&& f) {
#pragma unroll 4
    for (int32_t i = threadIdx.x * V; i < (int32_t)n; i += kClipThreads * V) f(i, i + V <= (int32_t)n);
}

// `once`: what is read is not kept in the caches.
template <typename T>
__device__ __forceinline__ double chunk_squares(const T* __restrict__ p, int64_t n, bool once) {
    constexpr int V = 16 / sizeof(T), U = kChunk / (kClipThreads * V);
    double s = 0.0;
    const auto add = [&](const Raw<V, T>& r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const double x = (double)(float)r.t[i];
            s += x * x;
        }
    };
    if (n == kChunk) {
        Raw<V, T> r[U];
        if (once)
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = load_raw_once<V>(p + (u * kClipThreads + threadIdx.x) * V);
        else
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = load_raw<V>(p + (u * kClipThreads + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) add(r[u]);
    } else {
        for_vectors<V>(n, [&](int32_t i, bool whole) {
            if (whole) {
                add(load_raw<V>(p + i));
            } else {
                for (; i < (int32_t)n; ++i) {
                    const double x = (double)(float)p[i];
                    s += x * x;
                }
            }
        });
    }
    return s;
}

template <typename S, typename D>
__device__ __forceinline__ void chunk_scale(const S* p, D* q, int64_t n, float f, float f2) {
    constexpr int V = 16 / (sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D)), U = kChunk / (kClipThreads * V);
    const auto put = [&](const Raw<V, S>& r, D* to) {
        float x[V];
        widen(r, x);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = x[i] * f2 * f;
        store_vec_once(to, x);
    };
    if (n == kChunk) {
        Raw<V, S> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_raw_once<V>(p + (u * kClipThreads + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) put(r[u], q + (u * kClipThreads + threadIdx.x) * V);
    } else {
        for_vectors<V>(n, [&](int32_t i, bool whole) {
            if (whole) {
                put(load_raw<V>(p + i), q + i);
            } else {
                for (; i < (int32_t)n; ++i) q[i] = (D)((float)p[i] * f2 * f);
            }
        });
    }
}

__global__ void __launch_bounds__(kClipThreads) k_clip_squares(Spans a, float keep, double* __restrict__ sums) {
    __shared__ double lds[kClipThreads / 64];
    const uint32_t c0 = (uint32_t)((uint64_t)a.chunks * blockIdx.x / gridDim.x);
    const uint32_t c1 = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / gridDim.x);
    const uint32_t kept = (uint32_t)((float)(c1 - c0) * keep);  // chunks that the second kernel will find in the caches
    double s = 0.0;
    uint32_t k = span_of(a, c0);
    for (uint32_t c = c0; c < c1; ++c) {
        const bool once = c < c1 - kept;
        while (k + 1 < a.count && a.s[k + 1].first <= c) ++k;
        const int64_t at = (int64_t)(c - a.s[k].first) * a.chunk, n = min((int64_t)a.chunk, a.s[k].n - at);
        const void* const p = a.s[k].src;
        if (a.s[k].st == SCD_F32)
            s += chunk_squares((const float*)p + at, n, once);
        else if (a.s[k].st == SCD_BF16)
            s += chunk_squares((const bf16*)p + at, n, once);
        else
            s += chunk_squares((const f16*)p + at, n, once);
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
    // From the last chunk back: what the first kernel read last is still in the caches.
    uint32_t k = span_of(a, c1 - 1);
    for (uint32_t c = c1; c-- > c0;) {
        while (a.s[k].first > c) --k;
        const Span& t = a.s[k];
        if (!t.dst || (t.dst == t.src && factor == 1.0)) continue;
        const int64_t at = (int64_t)(c - t.first) * a.chunk, n = min((int64_t)a.chunk, t.n - at);
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
    int64_t used = 0, total = 0, bytes = 0;
    for (int64_t i = 0; i < count; ++i) {
        const scd_span_t& t = spans[i];
        if (!type_bytes(t.src_type) || (t.dst_type != t.src_type && t.dst_type != SCD_F32))
            return fail(SCD_ERR_UNSUPPORTED, "span %lld: float32, bfloat16 or float16 into that type or float32", (long long)i);
        if (t.n < 0 || t.n > kMaxElements - total || (t.n > 0 && !t.src)) return fail(SCD_ERR_INVALID, "span %lld: bad size or null pointer", (long long)i);
        if (t.n > 0 && t.dst == t.src && t.dst_type != t.src_type) return fail(SCD_ERR_INVALID, "span %lld: in place the types must be the same", (long long)i);
        used += t.n > 0;
        total += t.n;
        bytes += t.n * type_bytes(t.src_type);
    }
    const int64_t launches = std::max<int64_t>(1, ceil_div(used, kSpans));
    if (launches > kMaxSums) return fail(SCD_ERR_UNSUPPORTED, "more than %lld spans", (long long)kMaxSums * kSpans);
    // Workgroups' sums: every launch gets the same share of the workspace.
    const int64_t most = std::min<int64_t>(kClipBlocks, kMaxSums / launches);
    // Small chunks where whole ones would leave CUs idle.
    const int64_t chunk = total < kChunk * kClipBlocks / 2 ? kChunk / 4 : kChunk;
    hipStream_t s = (hipStream_t)stream;
    double* const sums = (double*)workspace;
    Spans a;
    a.chunk = (uint32_t)chunk;
    // Up to kSpans spans a launch.  The second kernel's launches go through them backwards, as its workgroups go through
    // their chunks, so that what was read last is read first.
    const auto gather = [&](int64_t& i, int64_t launch) {  // the spans from the i-th on, without the empty ones
        a.count = (uint32_t)std::min<int64_t>(kSpans, used - launch * kSpans);
        a.chunks = 0;
        int64_t bytes = 0;
        for (uint32_t k = 0; k < a.count; ++i) {
            const scd_span_t& t = spans[i];
            if (t.n == 0) continue;
            a.s[k++] = Span{t.src, t.dst, t.n, a.chunks, (uint8_t)t.src_type, (uint8_t)t.dst_type, 0};
            a.chunks += (uint32_t)ceil_div(t.n, chunk);
            bytes += t.n * type_bytes(t.src_type);
        }
        return bytes;
    };
    uint32_t n_sums = 0;
    int64_t i = 0, left = bytes;
    for (int64_t g = 0; g * kSpans < used; ++g) {
        const int64_t here = gather(i, g);
        left -= here;
        const float keep = std::min(1.0f, std::max(0.0f, (float)(kKeepBytes - left) / (float)here));
        const uint32_t blocks = (uint32_t)std::min<int64_t>(most, a.chunks);
        k_clip_squares<<<blocks, kClipThreads, 0, s>>>(a, keep, sums + n_sums);
        n_sums += blocks;
    }
    i = count;
    for (int64_t g = launches - 1; g >= 0; --g) {
        for (int64_t k = std::min<int64_t>(kSpans, used - g * kSpans); k > 0; --i) k -= spans[i - 1].n > 0;
        int64_t from = i;
        gather(from, g);
        const uint32_t blocks = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(most, a.chunks));
        k_clip_scale<<<blocks, kClipThreads, 0, s>>>(a, sums, n_sums, max_norm, g == 0 ? norm : nullptr);
    }
    return launched("scd_clip_grads");
}

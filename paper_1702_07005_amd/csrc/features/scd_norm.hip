// scd_norm.hip -- layer norm over the columns of a matrix, and its gradients (gfx950).
//
// Forward: m = mean x, v = mean (x - m)^2, r = 1/sqrt(v + eps), y = (x - m) r w + b.
// Backward, h = (x - m) r, g = dy w:  dx = r (g - mean g - h mean(g h)), dw = sum_rows dy h, db = sum_rows dy.
//
// Both are bound by memory: the forward pass reads and writes the matrix once, the backward pass reads two and
// writes one.  A row stays in the registers of a group of lanes between its statistics and its result, so that it is
// read once and the variance is that of the centred values.  Groups walk the rows with a fixed stride; the
// backward pass keeps its share of dw and db in registers on the way, each workgroup writes its sums to the
// workspace in 32 bits, and a second kernel adds them in a fixed order.
//
// Measured: forward 32,768 x 2,048 (bf16) 49 us, 5.5 TB/s; backward 50,000 x 624 (fp32) 66 us, 5.7 TB/s, and 16,384 x 4,096
// (bf16) 76 us, 5.3 TB/s, of which the addition of the workgroups' sums takes 5.
#include <algorithm>

#include "scd_device.h"
#include "scd_feat.h"

namespace scd {
namespace feat {
namespace {

// The columns of a lane's NV vectors: vector j of lane l is the (l + j LPR)-th of the row.
template <int VEC, int NV, int LPR>
struct Columns {
    int32_t at[NV];
    int32_t skip[NV];  // leading columns that another lane counts; VEC where the row has no such vector
    __device__ __forceinline__ Columns(int32_t lane, int32_t dim) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int32_t k = lane + j * LPR;
            at[j] = vec_column<VEC>(k, dim, skip[j]);
            skip[j] = min(skip[j], VEC);
        }
    }
};

// The sums of K values over each group of LPR lanes.  Groups wider than a wave go through LDS; `turn` alternates
// from call to call, so that one barrier a call is enough.
template <int LPR, int THREADS, int K>
__device__ __forceinline__ void group_sums(float (&s)[K], float* lds, int turn) {
    if constexpr (LPR <= 64) {
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = group_sum<LPR>(s[k]);
    } else {
        constexpr int kWaves = LPR / 64;
        float* const mine = lds + turn * (THREADS / 64) * K + (threadIdx.x / LPR) * kWaves * K;
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = group_sum<64>(s[k]);
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) mine[threadIdx.x % LPR / 64 * K + k] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            s[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s[k] += mine[w * K + k];
        }
    }
}

template <int LPR, int THREADS>
constexpr int lds_words(int k) {
    return LPR <= 64 ? 1 : 2 * (THREADS / 64) * k;
}

template <typename T, typename P>
struct NormArgs {
    const T* x;
    int64_t xstride;
    int32_t rows;
    int32_t dim;
    const P* weight;
    const P* bias;
    float eps;
    T* y;
    int64_t ystride;
    float* mean;
    float* rstd;
};

// A large output goes past the caches (ONCE): 100,000 x 624 (fp32, 250 MB out) 98.4 us through them, 95.5 past them,
// 16,384 x 2,048 (bf16, 67 MB) 25.3 and 22.4; a smaller one is left there for its reader.
// With a pass that reads the output at once, both together take 4 to 10 % less through the caches at every size up to
// 256 MB: 12,288 x 2,048 (50 MB) 20.9 through and 17.8 past them alone, 35.6 and 38.5 with the reader, 24,576 x 2,048
// (101 MB) 38.2 and 35.8, 62.7 and 69.4.
constexpr int64_t kOnceOut = int64_t(64) << 20;

template <int VEC, int NV, int LPR, int THREADS, bool ONCE, typename T, typename P>
__global__ void __launch_bounds__(THREADS) k_norm(NormArgs<T, P> a) {
    __shared__ float lds[lds_words<LPR, THREADS>(2)];
    constexpr int kGroups = THREADS / LPR;
    const int32_t lane = threadIdx.x % LPR;
    const int64_t g = (int64_t)blockIdx.x * kGroups + threadIdx.x / LPR, step = (int64_t)gridDim.x * kGroups;
    const Columns<VEC, NV, LPR> col(lane, a.dim);
    const float inv = 1.0f / (float)a.dim;
    Raw<VEC, T> next[NV];
    Raw<VEC, P> w[NV], b[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) next[j] = load_raw<VEC>(a.x + min(g, (int64_t)a.rows - 1) * a.xstride + col.at[j]);
    if (a.weight)
#pragma unroll
        for (int j = 0; j < NV; ++j) w[j] = load_raw<VEC>(a.weight + col.at[j]);
    else
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[j].t[i] = (P)1.0f;
    if (a.bias)
#pragma unroll
        for (int j = 0; j < NV; ++j) b[j] = load_raw<VEC>(a.bias + col.at[j]);
    else
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) b[j].t[i] = (P)0.0f;
    // Every group of a workgroup takes as many turns, those past the last row on that row and without a result.
    for (int64_t r0 = (int64_t)blockIdx.x * kGroups; r0 < a.rows; r0 += step) {
        const int64_t r = r0 + threadIdx.x / LPR;
        float x[NV][VEC];
#pragma unroll
        for (int j = 0; j < NV; ++j) widen(next[j], x[j]);
        if (r0 + step < a.rows)
#pragma unroll
            for (int j = 0; j < NV; ++j) next[j] = load_raw<VEC>(a.x + min(r + step, (int64_t)a.rows - 1) * a.xstride + col.at[j]);
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[0] += i >= col.skip[j] ? x[j][i] : 0.0f;
        group_sums<LPR, THREADS, 1>(s, lds, 0);
        const float mean = s[0] * inv;
        s[0] = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                x[j][i] -= mean;
                s[0] += i >= col.skip[j] ? x[j][i] * x[j][i] : 0.0f;
            }
        group_sums<LPR, THREADS, 1>(s, lds, 1);
        const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
        if (r < a.rows) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float wj[VEC], bj[VEC], y[VEC];
                widen(w[j], wj);
                widen(b[j], bj);
#pragma unroll
                for (int i = 0; i < VEC; ++i) y[i] = x[j][i] * rstd * wj[i] + bj[i];
                if (col.skip[j] < VEC) put_vec<ONCE>(a.y + r * a.ystride + col.at[j], y);
            }
            if (lane == 0) {
                if (a.mean) a.mean[r] = mean;
                if (a.rstd) a.rstd[r] = rstd;
            }
        }
    }
}

// Rows too wide for the registers: a workgroup reads its row three times (from the caches after the first), element by
// element, which bounds it: 4,096 x 32,768 forward 458 us in bf16 (1.2 TB/s) and 404 in fp32 (2.7 TB/s); backward, where dw
// and db go through the workspace with every row, 800 (1.0 TB/s) and 990 (1.6 TB/s).
constexpr int kWideThreads = 1024;

template <typename T, typename P>
__global__ void __launch_bounds__(kWideThreads) k_norm_wide(NormArgs<T, P> a) {
    __shared__ float lds[lds_words<kWideThreads, kWideThreads>(1)];
    const float inv = 1.0f / (float)a.dim;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* const x = a.x + r * a.xstride;
        T* const y = a.y + r * a.ystride;
        float s[1] = {0.0f};
        for (int32_t c = threadIdx.x; c < a.dim; c += kWideThreads) s[0] += (float)x[c];
        group_sums<kWideThreads, kWideThreads, 1>(s, lds, 0);
        const float mean = s[0] * inv;
        s[0] = 0.0f;
        for (int32_t c = threadIdx.x; c < a.dim; c += kWideThreads) {
            const float d = (float)x[c] - mean;
            s[0] += d * d;
        }
        group_sums<kWideThreads, kWideThreads, 1>(s, lds, 1);
        const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
        for (int32_t c = threadIdx.x; c < a.dim; c += kWideThreads) {
            const float w = a.weight ? (float)a.weight[c] : 1.0f, b = a.bias ? (float)a.bias[c] : 0.0f;
            y[c] = (T)(((float)x[c] - mean) * rstd * w + b);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

// ---------------------------------------------------------------------------------------- backward

template <typename T, typename P>
struct NormGradArgs {
    const T* dy;
    int64_t gstride;
    const T* x;
    int64_t xstride;
    const float* mean;
    const float* rstd;
    int32_t rows;
    int32_t dim;
    const P* weight;
    T* dx;
    int64_t dstride;
    float* sums;  // [workgroups][2][dim] of dw and db, or null
    P* dw;        // not null with one workgroup: its sums are the results
    P* db;
};

// Where the three matrices take more than the caches hold (ONCE), they are read and written past them: 50,000 x 624
// (fp32, 374 MB) 71.8 us through the caches, 66.3 past them, 16,384 x 4,096 (bf16, 403 MB) 79.5 and 76.5; but
// 4,096 x 4,096 (101 MB), whose inputs the caches may hold, 24.8 and 30.4.
// On both sides of the limit: 10,922 x 4,096 (bf16, 268 MB) 57.5 and 55.8, 13,653 x 4,096 (336 MB) 68.6 and 66.3;
// 35,848 x 624 (fp32, 268 MB) 53.1 and 49.4, 44,810 x 624 (336 MB) 64.6 and 59.8; with a pass that reads dx at once 80 and
// 84, 98 and 101 (bf16), 70.8 and 70.5, 85.8 and 85.4 (fp32).
constexpr int64_t kOnceBytes = int64_t(288) << 20;

template <int VEC, int NV, int LPR, int THREADS, bool ONCE, typename T, typename P>
__global__ void __launch_bounds__(THREADS) k_norm_grad(NormGradArgs<T, P> a) {
    constexpr int kGroups = THREADS / LPR;
    constexpr int kElems = LPR * NV * VEC;
    __shared__ float lds[lds_words<LPR, THREADS>(2)];
    __shared__ float part[kGroups > 1 ? kGroups * kElems : 1];
    // The weights stay in registers, but not where a thread's share of the row leaves none for them: then each row reads
    // them from the caches.
    constexpr bool kWeights = NV * VEC <= 16;
    const int32_t lane = threadIdx.x % LPR;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const Columns<VEC, NV, LPR> col(lane, a.dim);
    const float inv = 1.0f / (float)a.dim;
    Raw<VEC, T> ndy[NV], nx[NV];
    Raw<VEC, P> w[NV];
    float nmean, nrstd, dw[NV][VEC] = {}, db[NV][VEC] = {};
    const auto fetch = [&](int64_t row) {
        row = min(row, (int64_t)a.rows - 1);
#pragma unroll
        for (int j = 0; j < NV; ++j) ndy[j] = fetch_raw<VEC, ONCE>(a.dy + row * a.gstride + col.at[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j) nx[j] = fetch_raw<VEC, ONCE>(a.x + row * a.xstride + col.at[j]);
        nmean = a.mean[row];
        nrstd = a.rstd[row];
    };
    fetch((int64_t)blockIdx.x * kGroups + threadIdx.x / LPR);
    const auto weights = [&](int j) {
        if (a.weight)
            w[j] = load_raw<VEC>(a.weight + col.at[j]);
        else
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[j].t[i] = (P)1.0f;
    };
    if (kWeights)
#pragma unroll
        for (int j = 0; j < NV; ++j) weights(j);
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * kGroups; r0 < a.rows; r0 += step, turn ^= 1) {
        const int64_t r = r0 + threadIdx.x / LPR;
        float dy[NV][VEC], h[NV][VEC], s[2] = {0.0f, 0.0f};
        const float mean = nmean, rstd = nrstd, here = r < a.rows ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            widen(ndy[j], dy[j]);
            widen(nx[j], h[j]);
        }
        if (r0 + step < a.rows) fetch(r + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float wj[VEC];
            if (!kWeights) weights(j);
            widen(w[j], wj);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                h[j][i] = (h[j][i] - mean) * rstd;
                if (here != 0.0f) {
                    dw[j][i] += dy[j][i] * h[j][i];
                    db[j][i] += dy[j][i];
                }
                dy[j][i] *= wj[i];
                s[0] += i >= col.skip[j] ? dy[j][i] : 0.0f;
                s[1] += i >= col.skip[j] ? dy[j][i] * h[j][i] : 0.0f;
            }
        }
        group_sums<LPR, THREADS, 2>(s, lds, turn);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
        if (r < a.rows) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) dy[j][i] = rstd * (dy[j][i] - c1 - h[j][i] * c2);
                if (col.skip[j] < VEC) put_vec<ONCE>(a.dx + r * a.dstride + col.at[j], dy[j]);
            }
        }
    }
    if (!a.sums && !a.dw) return;
    float* const sums = a.sums + (int64_t)blockIdx.x * 2 * a.dim;
    for (int which = 0; which < 2; ++which) {
        P* const result = which ? a.db : a.dw;
        if constexpr (kGroups > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    part[(threadIdx.x / LPR) * kElems + (lane + j * LPR) * VEC + i] = which ? db[j][i] : dw[j][i];
            __syncthreads();
            for (int e = threadIdx.x; e < kElems; e += THREADS) {
                int32_t again;
                const int32_t c = vec_column<VEC>(e / VEC, a.dim, again) + e % VEC;
                if (e % VEC < again) continue;
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < kGroups; ++k) s += part[k * kElems + e];
                if (a.dw)
                    result[c] = (P)s;
                else
                    sums[which * a.dim + c] = s;
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (col.skip[j] < VEC) {
                    if (a.dw)
                        store_vec(result + col.at[j], which ? db[j] : dw[j]);
                    else
                        store_vec(sums + which * a.dim + col.at[j], which ? db[j] : dw[j]);
                }
        }
    }
}

template <typename T, typename P>
__global__ void __launch_bounds__(kWideThreads) k_norm_grad_wide(NormGradArgs<T, P> a) {
    __shared__ float lds[lds_words<kWideThreads, kWideThreads>(2)];
    const float inv = 1.0f / (float)a.dim;
    float* const dw = a.sums ? a.sums + (int64_t)blockIdx.x * 2 * a.dim : nullptr;
    if (a.dw)  // before dx, which may lie in x's or dy's place; each thread its own columns, here and below
        for (int32_t c = threadIdx.x; c < a.dim; c += kWideThreads) {
            float sw = 0.0f, sb = 0.0f;
            for (int64_t r = 0; r < a.rows; ++r) {
                const float d = (float)a.dy[r * a.gstride + c];
                sw += d * (((float)a.x[r * a.xstride + c] - a.mean[r]) * a.rstd[r]);
                sb += d;
            }
            a.dw[c] = (P)sw;
            a.db[c] = (P)sb;
        }
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const T* const dy = a.dy + r * a.gstride;
        const T* const x = a.x + r * a.xstride;
        T* const dx = a.dx + r * a.dstride;
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s[2] = {0.0f, 0.0f};
        for (int32_t c = threadIdx.x; c < a.dim; c += kWideThreads) {
            const float d = (float)dy[c], h = ((float)x[c] - mean) * rstd, g = d * (a.weight ? (float)a.weight[c] : 1.0f);
            s[0] += g;
            s[1] += g * h;
            if (a.sums) {  // each thread its own columns
                const bool first = r == blockIdx.x;
                dw[c] = (first ? 0.0f : dw[c]) + d * h;
                dw[a.dim + c] = (first ? 0.0f : dw[a.dim + c]) + d;
            }
        }
        group_sums<kWideThreads, kWideThreads, 2>(s, lds, turn);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
        for (int32_t c = threadIdx.x; c < a.dim; c += kWideThreads) {
            const float h = ((float)x[c] - mean) * rstd, g = (float)dy[c] * (a.weight ? (float)a.weight[c] : 1.0f);
            dx[c] = (T)(rstd * (g - c1 - h * c2));
        }
    }
}

// dw and db: the workgroups' sums, 64 columns a workgroup, in kSlices interleaved parts that are added in order.
constexpr int kSlices = 16;

template <typename P>
__global__ void __launch_bounds__(64 * kSlices) k_norm_params(const float* __restrict__ sums, int32_t parts, int32_t dim,
                                                              P* __restrict__ dw, P* __restrict__ db) {
    __shared__ float lds[kSlices][64];
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x % 64, width = 2 * (int64_t)dim;
    const int32_t slice = threadIdx.x / 64;
    float s = 0.0f;
    if (c < width)
#pragma unroll 8
        for (int32_t p = slice; p < parts; p += kSlices) s += sums[p * width + c];
    lds[slice][threadIdx.x % 64] = s;
    __syncthreads();
    if (slice == 0 && c < width) {
#pragma unroll
        for (int k = 1; k < kSlices; ++k) s += lds[k][threadIdx.x];
        if (c < dim)
            dw[c] = (P)s;
        else
            db[c - dim] = (P)s;
    }
}

// ---------------------------------------------------------------------------------------- host

// Calls f(Int<VEC>, Int<NV>, Int<LPR>) with the smallest group that holds a row of `dim` elements of T, or returns
// false where none does.  A wave holds four vectors a lane, but in the backward pass, which keeps six values per element,
// of 16-bit elements three; and the widest rows take 512 threads there, which may have 256 registers each, and 1,024 in
// the forward pass.
template <typename T, bool GRAD, typename F>
bool with_group(int64_t dim, F&& f) {
    constexpr int V = 16 / sizeof(T);
    const int64_t vecs = ceil_div(dim, V);
    if (dim < V)
        f(Int<1>{}, Int<1>{}, Int<8>{});
    else if (vecs <= 4)
        f(Int<V>{}, Int<1>{}, Int<4>{});
    else if (vecs <= 8)
        f(Int<V>{}, Int<1>{}, Int<8>{});
    else if (vecs <= 16)
        f(Int<V>{}, Int<1>{}, Int<16>{});
    else if (vecs <= 32)
        f(Int<V>{}, Int<1>{}, Int<32>{});
    else if (vecs <= 64)
        f(Int<V>{}, Int<1>{}, Int<64>{});
    else if (vecs <= 128)
        f(Int<V>{}, Int<2>{}, Int<64>{});
    else if (vecs <= 192)
        f(Int<V>{}, Int<3>{}, Int<64>{});
    else if (vecs <= 256)
        f(Int<V>{}, Int<GRAD && V == 8 ? 1 : 4>{}, Int<GRAD && V == 8 ? 256 : 64>{});
    else if (vecs <= 512)
        f(Int<V>{}, Int<2>{}, Int<256>{});
    else if (vecs <= 1024)
        f(Int<V>{}, Int<2>{}, Int<512>{});
    else if (vecs <= 2048)
        f(Int<V>{}, Int<GRAD ? 4 : 2>{}, Int<GRAD ? 512 : 1024>{});
    else if constexpr (V == 4) {
        if (vecs > 4096) return false;
        f(Int<V>{}, Int<GRAD ? 8 : 4>{}, Int<GRAD ? 512 : 1024>{});
    } else {
        return false;
    }
    return true;
}

constexpr int kNormThreads = 256;   // a workgroup, where a row's group is not wider
constexpr int kBlocks = 2048;       // workgroups at most: eight to each CU
// The backward pass's, whose sums of dw and db go through memory: two to a CU, or one where a row takes 512 threads, whose
// registers fill the CU (8,192 x 8,192 in bf16: 89 us with two, 83 with one).
constexpr int kGradBlocks = 512;
constexpr int kGradBlocksWide = 256;

template <typename F>
void with_types(int32_t type, int32_t param, F&& f) {
    with_type(type, [&](auto t) {
        using T = decltype(t);
        if constexpr (sizeof(T) == 4)
            f(t, t);
        else
            param == SCD_F32 ? f(t, float{}) : f(t, t);
    });
}

int check_norm(int32_t type, int32_t param_type, int64_t rows, int64_t dim) {
    if (!type_bytes(type) || (param_type != type && param_type != SCD_F32))
        return fail(SCD_ERR_UNSUPPORTED, "layer norm takes float32, bfloat16 or float16 with parameters of that type or float32");
    if (rows < 0 || rows > kMaxRows || dim < 1 || dim > kMaxDim)
        return fail(SCD_ERR_INVALID, "bad sizes rows=%lld dim=%lld", (long long)rows, (long long)dim);
    return SCD_OK;
}

int64_t grad_blocks(int64_t rows) { return std::min<int64_t>(rows, kGradBlocks); }

// Up to this many rows for each group of a workgroup, one workgroup does it all, which saves the second launch: 9 rows of 851
// (bf16) 10.4 us with two launches, 7.0 with one.  A row of 512 threads takes longer than the launch (4 rows of 8,505 in
// fp32 27 us alone): there one row.  A call of one row needs no workspace, whatever its groups.
constexpr int64_t kTurnsAlone = 4;

int64_t grad_workspace(int64_t rows, int64_t dim) { return rows <= 1 ? 0 : grad_blocks(rows) * 2 * dim * 4; }

}  // namespace
}  // namespace feat
}  // namespace scd

using namespace scd::feat;

extern "C" int scd_layer_norm(const void* x, int32_t type, int64_t x_stride, int64_t rows, int64_t dim, const void* weight,
                              const void* bias, int32_t param_type, float eps, void* y, int64_t y_stride, float* mean,
                              float* rstd, void* stream) {
    if (int r = check_norm(type, param_type, rows, dim)) return r;
    if (!(eps >= 0.0f)) return fail(SCD_ERR_INVALID, "eps must be >= 0");
    if (x_stride < 0 || (y_stride < dim && rows > 1)) return fail(SCD_ERR_INVALID, "bad row stride");
    if (x == y && rows > 1 && x_stride != y_stride) return fail(SCD_ERR_INVALID, "in place the strides must be the same");
    if (rows == 0) return SCD_OK;
    if (!x || !y) return fail(SCD_ERR_INVALID, "null device pointer");
    hipStream_t s = (hipStream_t)stream;
    with_types(type, param_type, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        const NormArgs<T, P> a{(const T*)x, x_stride, (int32_t)rows, (int32_t)dim, (const P*)weight, (const P*)bias, eps, (T*)y, y_stride, mean, rstd};
        const bool fits = with_group<T, false>(dim, [&](auto vec, auto nv, auto lpr) {
            constexpr int VEC = decltype(vec)::value, NV = decltype(nv)::value, LPR = decltype(lpr)::value;
            constexpr int THREADS = LPR > kNormThreads ? LPR : kNormThreads;
            const int64_t blocks = std::min<int64_t>(kBlocks, ceil_div(rows, THREADS / LPR));
            if (rows * dim * (int64_t)sizeof(T) < kOnceOut)
                k_norm<VEC, NV, LPR, THREADS, false><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
            else
                k_norm<VEC, NV, LPR, THREADS, true><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
        });
        if (!fits) k_norm_wide<<<(uint32_t)std::min<int64_t>(kBlocks, rows), kWideThreads, 0, s>>>(a);
    });
    return launched("scd_layer_norm");
}

extern "C" int scd_layer_norm_grad_workspace(int64_t rows, int64_t dim, int64_t* bytes) {
    if (!bytes) return fail(SCD_ERR_INVALID, "bytes is null");
    *bytes = 0;
    if (int r = check_norm(SCD_F32, SCD_F32, rows, dim)) return r;
    *bytes = grad_workspace(rows, dim);
    return SCD_OK;
}

extern "C" int scd_layer_norm_grad(const void* grad, int64_t grad_stride, const void* x, int64_t x_stride, int32_t type,
                                   const float* mean, const float* rstd, int64_t rows, int64_t dim, const void* weight,
                                   int32_t param_type, void* dx, int64_t dx_stride, void* dweight, void* dbias,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
    if (int r = check_norm(type, param_type, rows, dim)) return r;
    if (grad_stride < 0 || x_stride < 0 || (dx_stride < dim && rows > 1)) return fail(SCD_ERR_INVALID, "bad row stride");
    if (rows > 1 && ((dx == grad && dx_stride != grad_stride) || (dx == x && dx_stride != x_stride)))
        return fail(SCD_ERR_INVALID, "in place the strides must be the same");
    if (!dweight != !dbias) return fail(SCD_ERR_INVALID, "dweight and dbias go together");
    if (rows > 0 && (!grad || !x || !mean || !rstd || !dx)) return fail(SCD_ERR_INVALID, "null device pointer");
    const int64_t need = dweight ? grad_workspace(rows, dim) : 0;
    if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need))
        return fail(SCD_ERR_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)need);
    hipStream_t s = (hipStream_t)stream;
    with_types(type, param_type, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        NormGradArgs<T, P> a{(const T*)grad, grad_stride, (const T*)x, x_stride, mean, rstd, (int32_t)rows, (int32_t)dim, (const P*)weight, (T*)dx, dx_stride, nullptr, nullptr, nullptr};
        int64_t blocks = 0;
        const auto share = [&](int64_t groups, int64_t most, int64_t turns) {  // the workgroups, and where their sums go
            const bool alone = rows <= turns * groups;
            blocks = alone && dweight ? 1 : std::min<int64_t>(most, ceil_div(rows, groups));
            a.dw = alone ? (P*)dweight : nullptr;
            a.db = alone ? (P*)dbias : nullptr;
            a.sums = alone || !dweight ? nullptr : (float*)workspace;
        };
        const bool fits = rows > 0 && with_group<T, true>(dim, [&](auto vec, auto nv, auto lpr) {
            constexpr int VEC = decltype(vec)::value, NV = decltype(nv)::value, LPR = decltype(lpr)::value;
            constexpr int THREADS = LPR > kNormThreads ? LPR : kNormThreads;
            share(THREADS / LPR, LPR >= 512 ? kGradBlocksWide : kGradBlocks, LPR >= 512 ? 1 : kTurnsAlone);
            if (rows * dim * 3 * (int64_t)sizeof(T) < kOnceBytes)
                k_norm_grad<VEC, NV, LPR, THREADS, false><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
            else
                k_norm_grad<VEC, NV, LPR, THREADS, true><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
        });
        if (rows > 0 && !fits) {
            share(1, kGradBlocks, 1);
            k_norm_grad_wide<<<(uint32_t)blocks, kWideThreads, 0, s>>>(a);
        }
        if (dweight && !a.dw)  // without rows: zeros
            k_norm_params<<<(uint32_t)ceil_div(2 * dim, 64), 64 * kSlices, 0, s>>>((const float*)workspace, (int32_t)blocks, (int32_t)dim, (P*)dweight, (P*)dbias);
    });
    return launched("scd_layer_norm_grad");
}

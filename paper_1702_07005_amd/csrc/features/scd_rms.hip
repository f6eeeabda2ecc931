// scd_rms.hip -- root-mean-square norm over the columns of a matrix, with the residual's addition and an output in 8 bits,
// and its gradient (gfx950).
//
// Forward: h = x + residual, rounded to the elements' type; r = 1/sqrt(mean h^2 + eps), y = h r w.  The norm is of the
// rounded h, which the caller keeps: the gradient reads it, and is that of the values that were used.
// In 8 bits: q = y / s in 32 bits, rounded, s = max |y| / 448 over the row or over groups of its columns.
// Backward, n = h r, g = dy w:  dh = r (g - n mean(g n)) (+ the residual's gradient), dw = sum_rows dy n.
//
// All are bound by memory: every matrix is read or written once.  A row stays in the registers of a group of lanes
// between its statistics and its result; groups walk the rows with a fixed stride and load the next row before they work
// on this one.  The backward pass keeps its share of dw in registers on the way, each workgroup writes its sums to the
// workspace in 32 bits, and a second kernel adds them in a fixed order.
//
// Measured: forward with residual 32,768 x 2,048 (bf16) 87 us, 6.2 TB/s; 16,384 x 4,096 (bf16) with residual into 8 bits 76
// us, 6.2 TB/s; backward with the residual's gradient 16,384 x 4,096 (bf16) 89 us, 6.0 TB/s, of which the addition of the
// workgroups' sums takes 4.  Rows that are read again: 4,096 x 32,768 (bf16) 130 us forward, 317 backward.
#include <algorithm>

#include "scd_device.h"
#include "scd_e4m3.h"
#include "scd_feat.h"
#include "scd_rows.h"

namespace scd {
namespace feat {
namespace {

template <typename T, typename P>
struct RmsArgs {
    const T* x;
    int64_t xstride;
    const T* res;  // or null
    int64_t rstride;
    int32_t rows;
    int32_t dim;
    const P* weight;
    float eps;
    int32_t group;   // columns of a scale, 0: the row
    int32_t scales;  // of a row
    void* y;         // of T, or of 8 bits
    int64_t ystride;
    float* scale;
    T* sum;  // x + res, not null with res
    int64_t sstride;
    float* rstd;
};

// The values of a vector in 8 bits, from the `skip`-th on.
template <int VEC>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&v)[VEC], int32_t skip) {
    if constexpr (VEC == 1) {
        *p = (uint8_t)e4m3_pack4(v[0], 0.0f, 0.0f, 0.0f);
    } else {
        uint32_t w[VEC / 4];
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) w[i] = e4m3_pack4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        if (skip == 0) {
            __builtin_memcpy(p, w, sizeof w);
        } else {  // the columns before may have another scale
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i >= skip) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
        }
    }
}

// max |x| over each group of LPR lanes; groups wider than a wave go through LDS as group_sums does.
template <int LPR, int THREADS>
__device__ __forceinline__ float row_max(float x, float* lds, int turn) {
    if constexpr (LPR <= 64) {
        return group_max<LPR>(x, LPR);
    } else {
        constexpr int kWaves = LPR / 64;
        float* const mine = lds + turn * (THREADS / 64) + (threadIdx.x / LPR) * kWaves;
        x = group_max<64>(x, 64);
        if (threadIdx.x % 64 == 0) mine[threadIdx.x % LPR / 64] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x = fmaxf(x, mine[w]);
        return x;
    }
}

// Waves a SIMD that registers are left for: in 8 bits three vectors of 16-bit elements would take two more than four waves have
// (32,768 x 2,560, bf16, residual, 97 us with four and 106 with three).
constexpr int rms_waves(int elems, int lpr, int threads, bool q) { return q && elems == 24 && lpr > 64 && threads == 256 ? 4 : 1; }

// Q: the output in 8 bits.  ONCE: large matrices are read and written past the caches.
template <int VEC, int NV, int LPR, int THREADS, bool Q, bool ONCE, typename T, typename P>
__global__ void __launch_bounds__(THREADS, rms_waves(VEC * NV, LPR, THREADS, Q)) k_rms(RmsArgs<T, P> a) {
    __shared__ float lds[lds_words<LPR, THREADS>(1)];
    constexpr int kGroups = THREADS / LPR;
    const int32_t lane = threadIdx.x % LPR;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const Columns<VEC, NV, LPR> col(lane, a.dim);
    const float inv = 1.0f / (float)a.dim;
    Raw<VEC, T> next[NV], more[NV];
    Raw<VEC, P> w[NV];
    const auto fetch = [&](int64_t row) {
        row = min(row, (int64_t)a.rows - 1);
#pragma unroll
        for (int j = 0; j < NV; ++j) next[j] = fetch_raw<VEC, ONCE>(a.x + row * a.xstride + col.at[j]);
        if (a.res)
#pragma unroll
            for (int j = 0; j < NV; ++j) more[j] = fetch_raw<VEC, ONCE>(a.res + row * a.rstride + col.at[j]);
    };
    fetch((int64_t)blockIdx.x * kGroups + threadIdx.x / LPR);
    if (a.weight)
#pragma unroll
        for (int j = 0; j < NV; ++j) w[j] = load_raw<VEC>(a.weight + col.at[j]);
    else
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[j].t[i] = (P)1.0f;
    int turn = 0;
    // Every group of a workgroup takes as many turns, those past the last row on that row and without a result.
    for (int64_t r0 = (int64_t)blockIdx.x * kGroups; r0 < a.rows; r0 += step) {
        const int64_t r = r0 + threadIdx.x / LPR;
        const bool here = r < a.rows;
        float h[NV][VEC];
#pragma unroll
        for (int j = 0; j < NV; ++j) widen(next[j], h[j]);
        if (a.res) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Raw<VEC, T> sum;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    sum.t[i] = (T)(h[j][i] + (float)more[j].t[i]);
                    h[j][i] = (float)sum.t[i];
                }
                if (LPR <= 64 && here && col.skip[j] < VEC) put_vec<ONCE>(a.sum + r * a.sstride + col.at[j], h[j]);
            }
        }
        if (r0 + step < a.rows) fetch(r + step);
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[0] += i >= col.skip[j] ? h[j][i] * h[j][i] : 0.0f;
        group_sums<LPR, THREADS, 1>(s, lds, turn);
        turn ^= 1;
        // Only now has every wave of a wider group read the row, whose last vector begins early, on columns that another wave
        // may have; and the sum may take an input's place.  (8,192 x 8,191, bf16, 110 us so and 107 with the sum written above;
        // in a group of one wave 32,768 x 2,048 would take 88 so and takes 87.)
        if (LPR > 64 && a.res && here)
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (col.skip[j] < VEC) put_vec<ONCE>(a.sum + r * a.sstride + col.at[j], h[j]);
        const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
        float most = 0.0f, part[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float wj[VEC];
            widen(w[j], wj);
            part[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                h[j][i] = h[j][i] * rstd * wj[i];
                if (Q) part[j] = fmaxf(part[j], i >= col.skip[j] ? fabsf(h[j][i]) : 0.0f);
            }
            if (Q) most = fmaxf(most, part[j]);
        }
        if constexpr (Q) {
            if (a.group == 0) {
                const float scale = e4m3_scale(row_max<LPR, THREADS>(most, lds, turn));
                turn ^= 1;
                if (here && lane == 0) a.scale[r] = scale;
                divide(h, scale);
            }
            const int lanes = min(a.group / VEC, LPR);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (a.group) {
                    const float scale = e4m3_scale(group_max<(LPR < 32 ? LPR : 32)>(part[j], lanes));
                    const int32_t c = (lane + j * LPR) * VEC;
                    if (here && c < a.dim && c % a.group == 0) a.scale[r * a.scales + c / a.group] = scale;
                    divide(h[j], scale);
                }
                if (here && col.skip[j] < VEC) store_e4m3<VEC>((uint8_t*)a.y + r * a.ystride + col.at[j], h[j], col.skip[j]);
            }
        } else if (here) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (col.skip[j] < VEC) put_vec<ONCE>((T*)a.y + r * a.ystride + col.at[j], h[j]);
        }
        if (here && lane == 0 && a.rstd) a.rstd[r] = rstd;
    }
}

// Rows too wide for the registers are read again from the caches: a workgroup takes a row, and each thread its vectors of V
// elements, kAtOnce of them loaded before the first is used.  As in vec_column, the last vector begins early, and its
// first `skip` columns, which another thread has, are neither counted nor written: where the output takes an input's
// place they may hold either.  Each thread reads again what it wrote itself.
constexpr int kAtOnce = 4;

// The columns of a thread's next vectors; from the row's end on, the last one with all its columns skipped.
template <int V, int APART>
struct Vectors {
    int32_t at[kAtOnce], skip[kAtOnce];
    __device__ __forceinline__ Vectors(int32_t c, int32_t dim) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            at[u] = min(c + u * APART, dim - V);
            skip[u] = min(c + u * APART - at[u], V);
        }
    }
};

template <int V, typename T>
__device__ __forceinline__ void store_from(T* p, int32_t skip, const float (&v)[V]) {
    if (skip == 0) {
        store_vec(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= skip) p[i] = (T)v[i];
    }
}

template <bool Q, typename T, typename P>
__global__ void __launch_bounds__(kWideThreads) k_rms_wide(RmsArgs<T, P> a) {
    constexpr int V = 16 / sizeof(T), kApart = kWideThreads * V, kStep = kAtOnce * kApart;
    __shared__ float lds[lds_words<kWideThreads, kWideThreads>(1)];
    const float inv = 1.0f / (float)a.dim;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* const x = a.x + r * a.xstride;
        const T* const res = a.res ? a.res + r * a.rstride : nullptr;
        T* const sum = a.sum ? a.sum + r * a.sstride : nullptr;
        const T* const kept = res ? sum : x;
        float s[1] = {0.0f};
        for (int32_t c = threadIdx.x * V; c < a.dim; c += kStep) {
            const Vectors<V, kApart> col(c, a.dim);
            Raw<V, T> rx[kAtOnce], rr[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) rx[u] = load_raw<V>(x + col.at[u]);
            if (res)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) rr[u] = load_raw<V>(res + col.at[u]);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                float h[V];
                widen(rx[u], h);
                if (res) {
#pragma unroll
                    for (int i = 0; i < V; ++i) h[i] = (float)(T)(h[i] + (float)rr[u].t[i]);
                    store_from(sum + col.at[u], col.skip[u], h);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += i >= col.skip[u] ? h[i] * h[i] : 0.0f;
            }
        }
        group_sums<kWideThreads, kWideThreads, 1>(s, lds, turn);
        turn ^= 1;
        const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
        // f(u, the results of the thread's u-th vector), all vectors of a step
        const auto results = [&](const Vectors<V, kApart>& col, auto&& f) {
            Raw<V, T> rx[kAtOnce];
            Raw<V, P> rw[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) rx[u] = load_raw<V>(kept + col.at[u]);
            if (a.weight)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) rw[u] = load_raw<V>(a.weight + col.at[u]);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                float y[V];
                widen(rx[u], y);
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = y[i] * rstd * (a.weight ? (float)rw[u].t[i] : 1.0f);
                f(u, y);
            }
        };
        const auto largest = [&](const float(&y)[V], int32_t skip) {
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) most = fmaxf(most, i >= skip ? fabsf(y[i]) : 0.0f);
            return most;
        };
        if constexpr (Q) {
            float scale = 0.0f;
            if (a.group == 0) {
                float most = 0.0f;
                for (int32_t c = threadIdx.x * V; c < a.dim; c += kStep) {
                    const Vectors<V, kApart> col(c, a.dim);
                    results(col, [&](int u, const float(&y)[V]) { most = fmaxf(most, largest(y, col.skip[u])); });
                }
                scale = e4m3_scale(row_max<kWideThreads, kWideThreads>(most, lds, turn));
                turn ^= 1;
                if (threadIdx.x == 0) a.scale[r] = scale;
            }
            uint8_t* const q = (uint8_t*)a.y + r * a.ystride;
            for (int32_t c0 = 0; c0 < a.dim; c0 += kStep) {  // all lanes of a wave go on to its groups' last one
                const int32_t c = c0 + threadIdx.x * V;
                const Vectors<V, kApart> col(c, a.dim);
                results(col, [&](int u, float(&y)[V]) {
                    if (a.group) {
                        scale = e4m3_scale(group_max<32>(largest(y, col.skip[u]), a.group / V));
                        const int32_t first = c + u * kApart;
                        if (first < a.dim && first % a.group == 0) a.scale[r * a.scales + first / a.group] = scale;
                    }
                    divide(y, scale);
                    if (col.skip[u] < V) store_e4m3<V>(q + col.at[u], y, col.skip[u]);
                });
            }
        } else {
            T* const out = (T*)a.y + r * a.ystride;
            for (int32_t c = threadIdx.x * V; c < a.dim; c += kStep) {
                const Vectors<V, kApart> col(c, a.dim);
                results(col, [&](int u, const float(&y)[V]) { store_from(out + col.at[u], col.skip[u], y); });
            }
        }
        if (threadIdx.x == 0 && a.rstd) a.rstd[r] = rstd;
    }
}

// ---------------------------------------------------------------------------------------- backward

template <typename T, typename P>
struct RmsGradArgs {
    const T* dy;
    int64_t gstride;
    const T* h;
    int64_t hstride;
    const T* res;  // the residual's gradient, or null
    int64_t rstride;
    const float* rstd;
    int32_t rows;
    int32_t dim;
    const P* weight;
    T* dh;
    int64_t dstride;
    float* sums;  // [workgroups][dim] of dw, or null
    P* dw;        // not null with one workgroup: its sums are the result
};

template <int VEC, int NV, int LPR, int THREADS, bool ONCE, typename T, typename P>
__global__ void __launch_bounds__(THREADS) k_rms_grad(RmsGradArgs<T, P> a) {
    constexpr int kGroups = THREADS / LPR;
    constexpr int kElems = LPR * NV * VEC;
    __shared__ float lds[lds_words<LPR, THREADS>(1)];
    __shared__ float part[kGroups > 1 ? kGroups * kElems : 1];
    // The weights stay in registers, but not where a thread's share of the row leaves none for them: then each row reads
    // them from the caches.
    constexpr bool kWeights = NV * VEC <= 16;
    const int32_t lane = threadIdx.x % LPR;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const Columns<VEC, NV, LPR> col(lane, a.dim);
    const float inv = 1.0f / (float)a.dim;
    Raw<VEC, T> ndy[NV], nh[NV], nres[NV];
    Raw<VEC, P> w[NV];
    float nrstd, dw[NV][VEC] = {};
    const auto fetch = [&](int64_t row) {
        row = min(row, (int64_t)a.rows - 1);
#pragma unroll
        for (int j = 0; j < NV; ++j) ndy[j] = fetch_raw<VEC, ONCE>(a.dy + row * a.gstride + col.at[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j) nh[j] = fetch_raw<VEC, ONCE>(a.h + row * a.hstride + col.at[j]);
        if (a.res)
#pragma unroll
            for (int j = 0; j < NV; ++j) nres[j] = fetch_raw<VEC, ONCE>(a.res + row * a.rstride + col.at[j]);
        nrstd = a.rstd[row];
    };
    // The next row is loaded before this one is worked on, but not where the threads' registers do not hold both.
    constexpr bool kAhead = THREADS <= 512;
    if (kAhead) fetch((int64_t)blockIdx.x * kGroups + threadIdx.x / LPR);
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
        const bool here = r < a.rows;
        if (!kAhead) fetch(r);
        const float rstd = nrstd;
        float g[NV][VEC], n[NV][VEC], res[NV][VEC], s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            widen(ndy[j], g[j]);
            widen(nh[j], n[j]);
            if (a.res)
                widen(nres[j], res[j]);
            else
#pragma unroll
                for (int i = 0; i < VEC; ++i) res[j][i] = 0.0f;
        }
        if (kAhead && r0 + step < a.rows) fetch(r + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float wj[VEC];
            if (!kWeights) weights(j);
            widen(w[j], wj);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                n[j][i] *= rstd;
                if (here) dw[j][i] += g[j][i] * n[j][i];
                g[j][i] *= wj[i];
                s[0] += i >= col.skip[j] ? g[j][i] * n[j][i] : 0.0f;
            }
        }
        group_sums<LPR, THREADS, 1>(s, lds, turn);
        const float c = s[0] * inv;
        if (here) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[j][i] = rstd * (g[j][i] - n[j][i] * c) + res[j][i];
                if (col.skip[j] < VEC) put_vec<ONCE>(a.dh + r * a.dstride + col.at[j], g[j]);
            }
        }
    }
    if (!a.sums && !a.dw) return;
    float* const sums = a.sums + (int64_t)blockIdx.x * a.dim;
    if constexpr (kGroups > 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) part[(threadIdx.x / LPR) * kElems + (lane + j * LPR) * VEC + i] = dw[j][i];
        __syncthreads();
        for (int e = threadIdx.x; e < kElems; e += THREADS) {
            int32_t again;
            const int32_t c = vec_column<VEC>(e / VEC, a.dim, again) + e % VEC;
            if (e % VEC < again) continue;
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < kGroups; ++k) s += part[k * kElems + e];
            if (a.dw)
                a.dw[c] = (P)s;
            else
                sums[c] = s;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (col.skip[j] < VEC) {
                if (a.dw)
                    store_vec(a.dw + col.at[j], dw[j]);
                else
                    store_vec(sums + col.at[j], dw[j]);
            }
    }
}

// Wide rows: dw by columns, before the row kernel, which may overwrite the inputs.  A thread takes a vector of columns and
// every gridDim.y-th row.
constexpr int kColumnThreads = 256;

template <typename T, typename P>
__global__ void __launch_bounds__(kColumnThreads) k_rms_columns(RmsGradArgs<T, P> a) {
    constexpr int V = 16 / sizeof(T);
    const int32_t k = blockIdx.x * kColumnThreads + threadIdx.x;
    int32_t skip;
    const int32_t c = vec_column<V>(k, a.dim, skip);
    if (skip >= V) return;
    float dw[V] = {};
    for (int64_t r0 = blockIdx.y; r0 < a.rows; r0 += (int64_t)gridDim.y * kAtOnce) {
        Raw<V, T> rg[kAtOnce], rh[kAtOnce];
        float rstd[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t r = min(r0 + (int64_t)u * gridDim.y, (int64_t)a.rows - 1);
            rg[u] = load_raw<V>(a.dy + r * a.gstride + c);
            rh[u] = load_raw<V>(a.h + r * a.hstride + c);
            rstd[u] = a.rstd[r];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (r0 + (int64_t)u * gridDim.y < a.rows)
#pragma unroll
                for (int i = 0; i < V; ++i) dw[i] += (float)rg[u].t[i] * ((float)rh[u].t[i] * rstd[u]);
    }
    if (a.dw)
        store_from(a.dw + c, skip, dw);
    else
        store_from(a.sums + (int64_t)blockIdx.y * a.dim + c, skip, dw);
}

template <typename T, typename P>
__global__ void __launch_bounds__(kWideThreads) k_rms_grad_wide(RmsGradArgs<T, P> a) {
    constexpr int V = 16 / sizeof(T), kApart = kWideThreads * V, kStep = kAtOnce * kApart;
    __shared__ float lds[lds_words<kWideThreads, kWideThreads>(1)];
    const float inv = 1.0f / (float)a.dim;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const float rstd = a.rstd[r];
        const T* const dy = a.dy + r * a.gstride;
        const T* const h = a.h + r * a.hstride;
        const T* const more = a.res ? a.res + r * a.rstride : nullptr;
        T* const dh = a.dh + r * a.dstride;
        // f(u, g, n) for the thread's vectors of a step
        const auto values = [&](const Vectors<V, kApart>& col, auto&& f) {
            Raw<V, T> rg[kAtOnce], rh[kAtOnce];
            Raw<V, P> rw[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) rg[u] = load_raw<V>(dy + col.at[u]);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) rh[u] = load_raw<V>(h + col.at[u]);
            if (a.weight)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) rw[u] = load_raw<V>(a.weight + col.at[u]);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                float g[V], n[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    n[i] = (float)rh[u].t[i] * rstd;
                    g[i] = (float)rg[u].t[i] * (a.weight ? (float)rw[u].t[i] : 1.0f);
                }
                f(u, g, n);
            }
        };
        float s[1] = {0.0f};
        for (int32_t c = threadIdx.x * V; c < a.dim; c += kStep) {
            const Vectors<V, kApart> col(c, a.dim);
            values(col, [&](int u, const float(&g)[V], const float(&n)[V]) {
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += i >= col.skip[u] ? g[i] * n[i] : 0.0f;
            });
        }
        group_sums<kWideThreads, kWideThreads, 1>(s, lds, turn);
        const float mean = s[0] * inv;
        for (int32_t c = threadIdx.x * V; c < a.dim; c += kStep) {
            const Vectors<V, kApart> col(c, a.dim);
            values(col, [&](int u, float(&g)[V], const float(&n)[V]) {
                float res[V] = {};
                if (more) load_vec(more + col.at[u], res);
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] = rstd * (g[i] - n[i] * mean) + res[i];
                if (col.skip[u] < V) store_from(dh + col.at[u], col.skip[u], g);
            });
        }
    }
}

// dw: the workgroups' sums, kAcross columns a workgroup, in kSlices interleaved parts that are added in order.
constexpr int kAcross = 32;
constexpr int kSlices = 16;

template <typename P>
__global__ void __launch_bounds__(kAcross * kSlices) k_rms_params(const float* __restrict__ sums, int32_t parts, int32_t dim, P* __restrict__ dw) {
    __shared__ float lds[kSlices][kAcross];
    const int32_t column = threadIdx.x % kAcross, c = blockIdx.x * kAcross + column, slice = threadIdx.x / kAcross;
    float s = 0.0f;
    if (c < dim)
#pragma unroll 8
        for (int32_t p = slice; p < parts; p += kSlices) s += sums[(int64_t)p * dim + c];
    lds[slice][column] = s;
    __syncthreads();
    if (slice == 0 && c < dim) {
#pragma unroll
        for (int k = 1; k < kSlices; ++k) s += lds[k][column];
        dw[c] = (P)s;
    }
}

// ---------------------------------------------------------------------------------------- host

constexpr int kRmsThreads = 256;  // a workgroup, where a row's group is not wider
// Workgroups at most.  Rows of a wave or less: 2 M x 16 (fp32, residual) 88 us with these, 92 with 8,192, 97 with 2,048 and
// 87 without a limit, but 2 M x 16 (bf16) 44.6, 44.3, 51 and 50; with 8 bits 50,000 x 624 (bf16) 40 with 8,192 and 44.
constexpr int64_t kRmsBlocksNarrow = 16384;
constexpr int64_t kRmsBlocks8 = 8192;
// Of 128 or 256 lanes: 16,384 x 4,096 (bf16, residual) 87 us with a workgroup for each row, 88 with 8,192, 94 with 2,048.
constexpr int64_t kRmsBlocks = 65536;
// Wider: 4,096 x 16,384 (bf16) 48 us with 2,048, 61 with a workgroup for each row; 8,192 x 8,192 45 and 46.5.
constexpr int64_t kRmsBlocksWide = 2048;
// The backward pass's, whose sums of dw go through memory: one to a CU.  16,384 x 4,096 (bf16) 72 us, with 512 workgroups of
// 256 threads 74, with 512 of 512 76; 4,099 x 1,000 (fp16) 9.3, 10.5 and 11.4.
constexpr int kRmsGradThreads = 512;
constexpr int kRmsGradBlocks = 256;
constexpr int64_t kColumnBlocks = 1024;  // of the sums by columns, which are at least nine across: fewer than 256 a column
// Rows for each group of a workgroup up to which one workgroup does it all, which saves the second launch; a row of 512
// threads or more takes longer than the launch: there one row.
constexpr int64_t kRmsTurnsAlone = 4;
// Bytes of all matrices from which they go past the caches.  Forward: 402 MB (12,288 x 4,096, bf16, residual) 65 us past
// them and 68 through them, 268 MB 44 and 41, 537 MB 86 and 90; with a pass that reads the output at once 97 and 91, 66 and
// 61, 127 and 135.  In 8 bits 352 MB 57 and 62, 235 MB 39 and 38.5.  Backward: 403 MB 75 and 78, 302 MB 58 and 58, 201 MB 42
// and 40; with a reader 114 and 126, 89 and 88, 63 and 61.
constexpr int64_t kRmsOnce = int64_t(384) << 20;
constexpr int64_t kRmsOnce8 = int64_t(288) << 20;
constexpr int64_t kRmsGradOnce = int64_t(320) << 20;

// Workgroups for `turns` turns, `most` of them at most, each with as many turns.
int64_t even_blocks(int64_t turns, int64_t most) { return ceil_div(turns, ceil_div(turns, most)); }

// with_group, but with three vectors a lane where two leave a quarter of twice the lanes or more without work: 8,000 x 10,000
// (bf16) 55 us and 60, 16,384 x 2,560 (fp32, residual) 108 and 121, into 8 bits 16,384 x 2,560 (bf16) 54 and 59; backward in
// fp32 alone, 16,384 x 2,500 85 and 92, for with 16-bit elements three vectors take registers that leave a SIMD two waves
// (16,384 x 2,560 57 and 48).  There groups of as many waves as two vectors a lane need: with the residual's gradient 16,384 x
// 5,120 121 and 129, 8,000 x 10,000 108 and 119, 8,192 x 12,288 116 and 128 (bf16); but of fourteen waves 4,096 x 14,336 89
// and 78, and forward or in fp32 no width gains by it.  The backward pass's widest rows take 1,024 threads that load a row
// when they come to it: 8,192 x 16,384 (bf16) 142 us, with 512 threads that load the next one ahead 169; 4,096 x 16,384
// (fp32) 149 and 229.  (These spill a few of their 128 registers, 6 to 16 with 16-bit elements and 27 in fp32.)
template <typename T, bool GRAD, typename F>
bool with_rms_group(int64_t dim, F&& f) {
    constexpr int V = 16 / sizeof(T);
    const int64_t vecs = ceil_div(dim, V);
    if constexpr (!GRAD || V == 4) {
        const bool narrow = vecs > 256 && vecs <= 3 * 128, wide = vecs > 512 && vecs <= 3 * 256, widest = vecs > 1024 && vecs <= 3 * 512;
        if (narrow) f(Int<V>{}, Int<3>{}, Int<128>{});
        if (wide) f(Int<V>{}, Int<3>{}, Int<256>{});
        if (widest) f(Int<V>{}, Int<3>{}, Int<512>{});
        if (narrow || wide || widest) return true;
    } else if (vecs > 512) {
        const int64_t waves = ceil_div(vecs, 128);
        if (waves == 5) f(Int<V>{}, Int<2>{}, Int<320>{});
        if (waves == 6) f(Int<V>{}, Int<2>{}, Int<384>{});
        if (waves == 7) f(Int<V>{}, Int<2>{}, Int<448>{});
        if (waves == 9 || waves == 10) f(Int<V>{}, Int<2>{}, Int<640>{});
        if (waves == 11 || waves == 12) f(Int<V>{}, Int<2>{}, Int<768>{});
        if (waves <= 12 && waves != 8) return true;
    }
    if constexpr (!GRAD) {
        return with_group<T, false>(dim, f);
    } else {
        if (vecs <= 1024)
            with_usual_group<T, true>(dim, f);
        else if (vecs <= 2048)
            f(Int<V>{}, Int<2>{}, Int<1024>{});
        else if (V == 4 && vecs <= 4096)
            f(Int<V>{}, Int<V == 4 ? 4 : 2>{}, Int<1024>{});
        else
            return false;
        return true;
    }
}

int check_rms(int32_t type, int32_t param_type, int64_t rows, int64_t dim) {
    if (!type_bytes(type) || (param_type != type && param_type != SCD_F32))
        return fail(SCD_ERR_UNSUPPORTED, "rms norm takes float32, bfloat16 or float16 with a weight of that type or float32");
    if (rows < 0 || rows > kMaxRows || dim < 1 || dim > kMaxDim)
        return fail(SCD_ERR_INVALID, "bad sizes rows=%lld dim=%lld", (long long)rows, (long long)dim);
    return SCD_OK;
}

int64_t rms_grad_workspace(int64_t rows, int64_t dim) { return rows <= 1 ? 0 : std::min<int64_t>(rows, kRmsGradBlocks) * dim * 4; }

}  // namespace
}  // namespace feat
}  // namespace scd

using namespace scd::feat;

extern "C" int scd_rms_norm(const void* x, int32_t type, int64_t x_stride, const void* residual, int64_t residual_stride, int64_t rows,
                            int64_t dim, const void* weight, int32_t param_type, float eps, void* y, int32_t y_type, int64_t y_stride,
                            float* scale, int64_t group, void* sum, int64_t sum_stride, float* rstd, void* stream) {
    if (int r = check_rms(type, param_type, rows, dim)) return r;
    if (y_type != type && y_type != SCD_E4M3) return fail(SCD_ERR_UNSUPPORTED, "rms norm gives its input's type or 8 bits (e4m3)");
    if (!(eps >= 0.0f)) return fail(SCD_ERR_INVALID, "eps must be >= 0");
    const bool eight = y_type == SCD_E4M3;
    if (eight ? group != 0 && group != 32 && group != 64 && group != 128 : group != 0)
        return fail(SCD_ERR_INVALID, "group must be 0 or, with 8 bits, 32, 64 or 128");
    if (x_stride < 0 || (residual && residual_stride < 0) || (rows > 1 && (y_stride < dim || (residual && sum_stride < dim))))
        return fail(SCD_ERR_INVALID, "bad row stride");
    if (rows == 0) return SCD_OK;
    if (!x || !y || (residual && !sum) || (eight && !scale)) return fail(SCD_ERR_INVALID, "null device pointer");
    if ((residual && sum == y) || (eight && (y == x || y == residual))) return fail(SCD_ERR_INVALID, "outputs overlap");
    if (rows > 1 && ((y == x && y_stride != x_stride) || (y == residual && y_stride != residual_stride) ||
                     (residual && ((sum == x && sum_stride != x_stride) || (sum == residual && sum_stride != residual_stride)))))
        return fail(SCD_ERR_INVALID, "in place the strides must be the same");
    hipStream_t s = (hipStream_t)stream;
    with_types(type, param_type, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        const RmsArgs<T, P> a{(const T*)x, x_stride, (const T*)residual, residual_stride, (int32_t)rows, (int32_t)dim, (const P*)weight, eps,
                              (int32_t)group, (int32_t)(group ? ceil_div(dim, group) : 1), y, y_stride, scale, residual ? (T*)sum : nullptr, sum_stride, rstd};
        const int64_t matrices = rows * dim * (int64_t)sizeof(T) * (residual ? 3 : 1);
        const bool once = eight ? matrices + rows * dim > kRmsOnce8 : matrices + rows * dim * (int64_t)sizeof(T) > kRmsOnce;
        const bool fits = with_rms_group<T, false>(dim, [&](auto vec, auto nv, auto lpr) {
            constexpr int VEC = decltype(vec)::value, NV = decltype(nv)::value, LPR = decltype(lpr)::value;
            constexpr int THREADS = LPR > kRmsThreads ? LPR : kRmsThreads;
            const uint32_t blocks = (uint32_t)even_blocks(ceil_div(rows, THREADS / LPR), LPR > 256 ? kRmsBlocksWide : LPR > 64 ? kRmsBlocks : eight ? kRmsBlocks8 : kRmsBlocksNarrow);
            if (eight)
                once ? k_rms<VEC, NV, LPR, THREADS, true, true><<<blocks, THREADS, 0, s>>>(a) : k_rms<VEC, NV, LPR, THREADS, true, false><<<blocks, THREADS, 0, s>>>(a);
            else
                once ? k_rms<VEC, NV, LPR, THREADS, false, true><<<blocks, THREADS, 0, s>>>(a) : k_rms<VEC, NV, LPR, THREADS, false, false><<<blocks, THREADS, 0, s>>>(a);
        });
        const uint32_t blocks = (uint32_t)std::min<int64_t>(kRmsBlocksWide, rows);
        if (!fits) eight ? k_rms_wide<true><<<blocks, kWideThreads, 0, s>>>(a) : k_rms_wide<false><<<blocks, kWideThreads, 0, s>>>(a);
    });
    return launched("scd_rms_norm");
}

extern "C" int scd_rms_norm_grad_workspace(int64_t rows, int64_t dim, int64_t* bytes) {
    if (!bytes) return fail(SCD_ERR_INVALID, "bytes is null");
    *bytes = 0;
    if (int r = check_rms(SCD_F32, SCD_F32, rows, dim)) return r;
    *bytes = rms_grad_workspace(rows, dim);
    return SCD_OK;
}

extern "C" int scd_rms_norm_grad(const void* grad, int64_t grad_stride, const void* h, int64_t h_stride, int32_t type, const float* rstd,
                                 int64_t rows, int64_t dim, const void* weight, int32_t param_type, const void* residual_grad,
                                 int64_t residual_stride, void* dh, int64_t dh_stride, void* dweight, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
    if (int r = check_rms(type, param_type, rows, dim)) return r;
    if (grad_stride < 0 || h_stride < 0 || (residual_grad && residual_stride < 0) || (dh_stride < dim && rows > 1))
        return fail(SCD_ERR_INVALID, "bad row stride");
    if (rows > 1 && ((dh == grad && dh_stride != grad_stride) || (dh == h && dh_stride != h_stride) ||
                     (residual_grad && dh == residual_grad && dh_stride != residual_stride)))
        return fail(SCD_ERR_INVALID, "in place the strides must be the same");
    if (rows == 0 && !dweight) return SCD_OK;
    if (rows > 0 && (!grad || !h || !rstd || !dh)) return fail(SCD_ERR_INVALID, "null device pointer");
    const int64_t need = dweight ? rms_grad_workspace(rows, dim) : 0;
    if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need))
        return fail(SCD_ERR_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)need);
    hipStream_t s = (hipStream_t)stream;
    with_types(type, param_type, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        RmsGradArgs<T, P> a{(const T*)grad, grad_stride, (const T*)h, h_stride, (const T*)residual_grad, residual_stride, rstd, (int32_t)rows,
                            (int32_t)dim, (const P*)weight, (T*)dh, dh_stride, nullptr, nullptr};
        int64_t blocks = 0;  // whose sums go through the workspace
        const bool fits = rows > 0 && with_rms_group<T, true>(dim, [&](auto vec, auto nv, auto lpr) {
            constexpr int VEC = decltype(vec)::value, NV = decltype(nv)::value, LPR = decltype(lpr)::value;
            constexpr int THREADS = LPR > kRmsGradThreads ? LPR : kRmsGradThreads / LPR * LPR;
            constexpr int64_t groups = THREADS / LPR;
            const bool alone = rows <= (LPR >= 512 ? 1 : kRmsTurnsAlone) * groups;
            blocks = alone && dweight ? 1 : std::min<int64_t>(kRmsGradBlocks, ceil_div(rows, groups));
            a.dw = alone ? (P*)dweight : nullptr;
            a.sums = alone || !dweight ? nullptr : (float*)workspace;
            if (rows * dim * (residual_grad ? 4 : 3) * (int64_t)sizeof(T) <= kRmsGradOnce)
                k_rms_grad<VEC, NV, LPR, THREADS, false><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
            else
                k_rms_grad<VEC, NV, LPR, THREADS, true><<<(uint32_t)blocks, THREADS, 0, s>>>(a);
        });
        if (rows > 0 && !fits) {
            if (dweight) {
                const int64_t across = ceil_div(dim, kColumnThreads * (16 / (int64_t)sizeof(T)));
                blocks = std::min<int64_t>(rows, std::max<int64_t>(1, kColumnBlocks / across));
                a.dw = blocks == 1 ? (P*)dweight : nullptr;
                a.sums = (float*)workspace;
                k_rms_columns<<<dim3((uint32_t)across, (uint32_t)blocks), kColumnThreads, 0, s>>>(a);
            }
            k_rms_grad_wide<<<(uint32_t)std::min<int64_t>(kRmsBlocksWide, rows), kWideThreads, 0, s>>>(a);
        }
        if (dweight && !a.dw)  // without rows: zeros
            k_rms_params<<<(uint32_t)ceil_div(dim, kAcross), kAcross * kSlices, 0, s>>>((const float*)workspace, (int32_t)blocks, (int32_t)dim, (P*)dweight);
    });
    return launched("scd_rms_norm_grad");
}

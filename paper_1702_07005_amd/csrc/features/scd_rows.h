// scd_rows.h -- what the norms (scd_norm.hip, scd_rms.hip) share: rows held in the registers of a group of lanes, the sums
// over such a group, and the choice of the group by a row's width.
#pragma once

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

// Rows too wide for the registers: threads of the workgroup that takes one.
constexpr int kWideThreads = 1024;

// ---------------------------------------------------------------------------------------- host

// Calls f(Int<VEC>, Int<NV>, Int<LPR>) with the smallest group that holds a row of `dim` elements of T, 1,024 vectors at most.
// A wave holds four vectors a lane, but in the backward pass, which keeps six values per element, of 16-bit elements three.
template <typename T, bool GRAD, typename F>
void with_usual_group(int64_t dim, F&& f) {
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
    else
        f(Int<V>{}, Int<2>{}, Int<512>{});
}

// The same for rows of any width, or returns false where no group holds one.  The widest rows take 512 threads in the backward
// pass, which may have 256 registers each, and 1,024 in the forward pass.
template <typename T, bool GRAD, typename F>
bool with_group(int64_t dim, F&& f) {
    constexpr int V = 16 / sizeof(T);
    const int64_t vecs = ceil_div(dim, V);
    if (vecs <= 1024)
        with_usual_group<T, GRAD>(dim, f);
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

}  // namespace
}  // namespace feat
}  // namespace scd

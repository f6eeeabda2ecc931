// scd_feat.h -- what the operators of learned features (scd_embed.hip, scd_norm.hip, scd_clip.hip)
// share: element types, vectors of elements in registers, and the checks of their entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "scd.h"
#include "scd_kernels.h"
#include "scd_plan.h"

namespace scd {
namespace feat {

using bf16 = __bf16;
using f16 = _Float16;

// N consecutive elements as they are stored.  Rows may start at any element (odd widths, views), so the
// address is aligned to the element only; gfx950 loads and stores 16 bytes at such addresses in one access.
// Loading and widening are apart so that several loads can be in flight.
template <int N, typename T>
struct Raw {
    T t[N];
};

template <int N, typename T>
__device__ __forceinline__ Raw<N, T> load_raw(const T* __restrict__ p) {
    Raw<N, T> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}

template <int N, typename T>
__device__ __forceinline__ void widen(const Raw<N, T>& r, float (&o)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = (float)r.t[i];
}

template <int N, typename T>
__device__ __forceinline__ void load_vec(const T* __restrict__ p, float (&o)[N]) {
    widen(load_raw<N>(p), o);
}

template <int N, typename T>
__device__ __forceinline__ void store_vec(T* __restrict__ p, const float (&v)[N]) {
    Raw<N, T> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.t[i] = (T)v[i];
    __builtin_memcpy(p, &r, sizeof r);
}

// The same past the caches (non-temporal): for data that is touched once and larger than what the caches would keep.
template <int BYTES>
struct Words {
    typedef uint32_t type __attribute__((ext_vector_type(BYTES / 4), aligned(2)));
};
template <>
struct Words<2> {
    typedef uint16_t type;
};
template <>
struct Words<4> {
    typedef uint32_t type __attribute__((aligned(2)));
};

template <int N, typename T>
__device__ __forceinline__ Raw<N, T> load_raw_once(const T* __restrict__ p) {
    using W = typename Words<sizeof(Raw<N, T>)>::type;
    const W w = __builtin_nontemporal_load(reinterpret_cast<const W*>(p));
    return __builtin_bit_cast(Raw<N, T>, w);
}

template <int N, typename T>
__device__ __forceinline__ void store_vec_once(T* __restrict__ p, const float (&v)[N]) {
    using W = typename Words<sizeof(Raw<N, T>)>::type;
    Raw<N, T> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.t[i] = (T)v[i];
    __builtin_nontemporal_store(__builtin_bit_cast(W, r), reinterpret_cast<W*>(p));
}

template <int N, bool ONCE, typename T>
__device__ __forceinline__ Raw<N, T> fetch_raw(const T* __restrict__ p) {
    if constexpr (ONCE)
        return load_raw_once<N>(p);
    else
        return load_raw<N>(p);
}

template <bool ONCE, int N, typename T>
__device__ __forceinline__ void put_vec(T* __restrict__ p, const float (&v)[N]) {
    if constexpr (ONCE)
        store_vec_once(p, v);
    else
        store_vec(p, v);
}

// Vectors of a row: the k-th begins at column k N, except the last of a width that N does not divide, which
// begins at dim - N instead and repeats `again` columns of the one before it.  Every vector is whole (dim >= N),
// so there is no code for tails; what is computed per column comes out the same in both, and sums over
// columns leave the repeated ones out.
template <int N>
__device__ __forceinline__ int32_t vec_column(int32_t k, int32_t dim, int32_t& again) {
    const int32_t c = k * N, last = dim - N;
    again = c > last ? c - last : 0;
    return c > last ? last : c;
}

inline int type_bytes(int32_t t) { return t == SCD_F32 ? 4 : t == SCD_BF16 || t == SCD_F16 ? 2 : 0; }

// Records the message that scd_last_error returns on this thread.
inline int fail(int code, const char* fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        set_last_error(buf);
    } catch (...) {  // no memory for the message: the status alone is returned
    }
    return code;
}

inline int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SCD_OK : fail(SCD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f with a value of the element type, so that f can be a generic lambda.
template <typename F>
inline void with_type(int32_t t, F&& f) {
    if (t == SCD_F32)
        f(float{});
    else if (t == SCD_BF16)
        f(bf16{});
    else
        f(f16{});
}

constexpr int64_t kMaxDim = int64_t(1) << 20;
constexpr int64_t kMaxRows = 2147483647LL;

}  // namespace feat
}  // namespace scd

// scd_adamw.hip -- one AdamW step over many tensors, with states in 32 bits or in 8 (gfx950).
//
// g = f grad, f = max_norm / norm if norm > max_norm else 1;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;
// p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps);  copy = p rounded.
//
// Bound by memory: every tensor is read once and written once.  The tensors' addresses travel in the launch's arguments
// (up to kSteps a launch), so that a call copies nothing to the GPU; a tensor is cut into chunks, a workgroup for each.
// Launches do not depend on one another, and no element on another one but for the scales.
//
// In 8 bits (e4m3) a block of 256 elements has one scale for m and one for r = sqrt(v): the square root halves the range of
// exponents that v would need.  A wave takes two blocks, eight elements a lane.  States are rounded up or down at random: to
// the nearest, v, which moves by a thousandth of itself in a step where half a step of its 8 bits is 6 to 12 %, would never
// move again.  m goes up with the probability that keeps its mean, r with the one that keeps the mean of r^2; r > 0 never
// becomes 0, where m over it would be without bound.  The random numbers are a hash of seed, step, tensor and element.
//
// Measured: 354 M weights (fp32, gradients and copies in bf16) 1,543 us with states of 32 bits, 6.4 TB/s of the 9.9 GB that
// it cannot do without, and 909 us with 8, 6.3 TB/s of 5.7 GB, where the arithmetic (77 instructions an element) keeps the
// SIMDs busy for two thirds of that time; 11 tensors of 160,000 weights in all 3.8 and 4.7 us on the GPU.
#include <algorithm>
#include <cmath>

#include "scd_device.h"
#include "scd_e4m3.h"
#include "scd_feat.h"

namespace scd {
namespace feat {
namespace {

constexpr int kSteps = 64;             // tensors a launch, a lane for each: the arguments stay below 4 KB
constexpr int kSteps8 = 47;            // with states of 8 bits
constexpr int kStateBlock = 256;       // elements that share a scale
// A workgroup is one wave, and has one turn.  In this order, what runs at a time lies close together in memory: 354 M weights
// 2,011 us with 2,048 workgroups of 256 threads that each take a run of chunks, 1,692 with a workgroup of 256 for each 1,024
// elements, 1,640 with one of 64 for each 256 (states of 32 bits); with 8 bits 1,191, 980 and 960.
constexpr int kStepThreads = 64;
constexpr int64_t kStepChunk = 256;    // elements of a workgroup, 32 bits
// There a tensor's chunks begin where its states' lines do, the first of them up to this many elements early: tensors at odd
// places of one buffer (26 layers of width 897, 107 M weights in all, fp32 gradients, bf16 copies) 515 us, without this 708,
// of width 896 502.
constexpr uint32_t kStepLine = 64;
// With 8 bits, where the blocks are fixed, as many consecutive chunks go to one XCD, so that few lines are shared between two:
// 354 M weights 914 us, 966 without; 945 with 256, 983 with 16.  With 32 bits 1,693 with 64 and 1,555 without.
constexpr uint32_t kTogether8 = 64;
constexpr uint32_t kXcds = 8;
constexpr int64_t kStepChunk8 = 512;   // and 8
constexpr int64_t kStepBlocks = kMaxThreads / kStepThreads;  // workgroups of a launch at most
constexpr int64_t kStepMost = int64_t(1) << 39;              // elements of a call: chunk numbers stay below 2^32
// Calls that read and write this much go past the caches.  On states that other work has displaced: 10 M weights (280 MB, 32
// bits) 47 us past them and 54 through them, 6 M (168 MB) 30 and 35, 1 M (28 MB) 7.1 and 7.2; with a pass that reads the
// copy at once 60 and 62, 40 and 40, 10.8 and 10.2; but on states that the caches still hold 6 M take 29 and 27.  Not where
// the accesses are not of whole lines, which are then read and written twice: with 8 bits and width 897 348 us through the
// caches, 387 past them (bf16 gradients), of width 896 324 and 290.
constexpr int64_t kStepOnce = int64_t(128) << 20;
// LDS that a workgroup of states in 32 bits asks for and does not use, so that sixteen are on a CU at a time, four to a SIMD:
// with fewer bytes in flight the memory gives more.  354 M weights: 32 waves 1,645 us, 20 1,556, 16 1,548, 14 1,558, 12
// 1,597, 8 1,976.  States of 8 bits, whose waves compute as long as they wait, take as many as their registers allow.
constexpr int kStepLds = 10240;

struct Step32 {
    void* p;
    const void* g;
    void* m;
    void* v;
    void* copy;
    int64_t n;
    float decay;
    uint8_t pt, gt, ct, pad_;
};
struct Step8 {
    void* p;
    const void* g;
    void* m;
    void* v;
    void* copy;
    int64_t n;
    float decay;
    uint8_t pt, gt, ct, pad_;
    float* ms;
    float* vs;
    uint64_t place;  // in the call's list
};
template <bool EIGHT>
struct StepArgs {
    static constexpr int kMost = EIGHT ? kSteps8 : kSteps;
    std::conditional_t<EIGHT, Step8, Step32> s[kMost];
    uint32_t first[kMost];  // number of chunks before each tensor's
    uint32_t count;
    uint32_t chunks;
    uint32_t from;  // the launch's first chunk
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* norm_dev;
    int64_t step;
    double lr;
    double log_b1, log_b2;
    float b1, b2, a1, a2;  // a = 1 - b
    float eps, max_norm;
    float rate, root;  // where neither lr nor step are on the GPU
};
static_assert(sizeof(StepArgs<false>) <= 4096 && sizeof(StepArgs<true>) <= 4096, "kernel arguments");
static_assert(kSteps <= 64 && kSteps8 <= 64, "a lane for each tensor");

// The elements by which a tensor's first chunk begins early.
template <bool EIGHT>
__host__ __device__ inline uint32_t early(const void* m) {
    return EIGHT ? 0 : (uint32_t)((uintptr_t)m / 4 % kStepLine);
}

// What all elements of a launch share.
struct Common {
    float f, b1, b2, a1, a2, eps;
    float rate;  // lr / (1 - b1^t)
    float root;  // 1 / sqrt(1 - b2^t)
    double lr;
    uint32_t key;
};

template <bool EIGHT>
__device__ __forceinline__ Common common_of(const StepArgs<EIGHT>& a) {
    Common c;
    c.b1 = a.b1;
    c.b2 = a.b2;
    c.a1 = a.a1;
    c.a2 = a.a2;
    c.eps = a.eps;
    c.f = 1.0f;
    if (a.norm_dev) {
        const float norm = *a.norm_dev;
        c.f = norm <= a.max_norm ? 1.0f : a.max_norm / norm;  // NaN: NaN
    }
    c.lr = a.lr;
    c.rate = a.rate;
    c.root = a.root;
    int64_t t = a.step;
    if (a.step_dev || a.lr_dev) {
        if (a.step_dev) t = max(*a.step_dev, (int64_t)1);
        if (a.lr_dev) c.lr = (double)*a.lr_dev;
        // 1 - b^t without cancellation
        c.rate = (float)(c.lr / -expm1((double)t * a.log_b1));
        c.root = (float)(1.0 / sqrt(-expm1((double)t * a.log_b2)));
    }
    c.key = murmur_fmix32(a.seed ^ murmur_fmix32((uint32_t)t));
    return c;
}

// The tensor that holds a chunk: a lane looks at each.
template <bool EIGHT>
__device__ __forceinline__ uint32_t tensor_of(const StepArgs<EIGHT>& a, uint32_t chunk) {
    const uint32_t lane = threadIdx.x % 64;
    const uint64_t before = __ballot(lane < a.count && a.first[min(lane, (uint32_t)a.kMost - 1)] <= chunk);
    return (uint32_t)__builtin_popcountll(before) - 1;
}

template <bool ONCE, int V>
__device__ __forceinline__ void store_copy(void* copy, int32_t type, int64_t i, const float (&p)[V]) {
    if (type == SCD_BF16)
        put_vec<ONCE>((bf16*)copy + i, p);
    else
        put_vec<ONCE>((f16*)copy + i, p);
}

template <bool ONCE, int V, typename T>
__device__ __forceinline__ void fetch_vec(const T* p, float (&o)[V]) {
    widen(fetch_raw<V, ONCE>(p), o);
}

// Four values of 8 bits.
typedef uint32_t Four __attribute__((aligned(1)));
template <bool ONCE>
__device__ __forceinline__ uint32_t fetch_4(const uint8_t* p) {
    return ONCE ? __builtin_nontemporal_load((const Four*)p) : *(const Four*)p;
}
template <bool ONCE>
__device__ __forceinline__ void put_4(uint8_t* p, uint32_t w) {
    if (ONCE)
        __builtin_nontemporal_store(w, (Four*)p);
    else
        *(Four*)p = w;
}

// V elements from the i-th on, states in 32 bits.
template <bool ONCE, int V, typename P, typename G>
__device__ __forceinline__ void step_32(const Common& c, const Step32& s, float keep, int64_t i) {
    float p[V], g[V], m[V], v[V];
    fetch_vec<ONCE>((const P*)s.p + i, p);
    fetch_vec<ONCE>((const G*)s.g + i, g);
    fetch_vec<ONCE>((const float*)s.m + i, m);
    fetch_vec<ONCE>((const float*)s.v + i, v);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        g[k] *= c.f;
        m[k] = c.b1 * m[k] + c.a1 * g[k];
        v[k] = c.b2 * v[k] + c.a2 * (g[k] * g[k]);
        p[k] = p[k] * keep - c.rate * m[k] / (sqrtf(v[k]) * c.root + c.eps);
    }
    put_vec<ONCE>((P*)s.p + i, p);
    put_vec<ONCE>((float*)s.m + i, m);
    put_vec<ONCE>((float*)s.v + i, v);
    if (s.copy) store_copy<ONCE>(s.copy, s.ct, i, p);
}

// A wave's chunk, four elements a lane; one that the tensor fills in part goes element by element.
template <bool ONCE, typename P, typename G>
__device__ __forceinline__ void chunk_32(const Common& c, const Step32& s, int64_t at) {
    static_assert(kStepChunk == kStepThreads * 4, "one turn");
    const float keep = (float)(1.0 - c.lr * (double)s.decay);
    if (at >= 0 && at + kStepChunk <= s.n) {
        step_32<ONCE, 4, P, G>(c, s, keep, at + threadIdx.x * 4);
    } else {
        const int64_t end = min(at + kStepChunk, s.n);
        for (int64_t k = max(at, (int64_t)0) + threadIdx.x; k < end; k += kStepThreads) step_32<false, 1, P, G>(c, s, keep, k);
    }
}

constexpr uint32_t kLargest = 0x7F7FFFFFu;  // bits of the largest finite number
constexpr float kSmallRoot = 0x1p-96f;

// The averages of a state in 8 bits.  Every product and sum rounds by itself, divide() and root() below as a division and a
// square root do, and the scale is the product that the header states: a state that lies at the border between up and down
// goes the same way wherever these formulas are computed in 32 bits.
__device__ __forceinline__ void next_moments(const Common& c, float g, float m0, float r0, float& m, float& v) {
#pragma clang fp contract(off)
    m = c.b1 * m0 + c.a1 * g;
    v = c.b2 * (r0 * r0) + c.a2 * (g * g);
}

// sqrt(v), rounded once, of 0 or v >= 2^-96.  The instruction's result s is a unit off at most; with its neighbour d below, s d
// is the square of the point between them but for a quarter of a unit squared, so that v <= s d says that d is nearer.
__device__ __forceinline__ float root(float v) {
    const float s = __builtin_amdgcn_sqrtf(v);
    const float down = __uint_as_float(__float_as_uint(s) - 1), up = __uint_as_float(__float_as_uint(s) + 1);
    const float lower = fmaf(-down, s, v) <= 0.0f ? down : s;
    return fmaf(-up, s, v) > 0.0f ? up : lower;
}

// The largest of the bits of numbers >= 0, whose order is that of the numbers, over 32 lanes; a NaN is above all.
__device__ __forceinline__ uint32_t block_most(uint32_t x) {
    const auto dpp = [](uint32_t y, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)y, decltype(ctrl)::value, 0xF, 0xF, false); };
    x = max(x, dpp(x, Int<0xB1>{}));   // lane ^ 1
    x = max(x, dpp(x, Int<0x4E>{}));   // lane ^ 2
    x = max(x, dpp(x, Int<0x141>{}));  // other quad of 8
    x = max(x, dpp(x, Int<0x140>{}));  // other half of 16
    return max(x, (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401F));  // lane ^ 16
}

// What the conversion adds for a word: 2^16 - 1 less its low half, and 7 sixteenths.
__device__ __forceinline__ uint32_t random_bits(uint32_t word) { return (~word << 16) | 0x7000u; }

// Four values in 8 bits, up or down with the random numbers of the words' low halves: the instruction adds its operand's 20
// upper bits below the last bit that stays and cuts off.  It goes away from 0 where the fraction, of 20 bits, is above
// (word mod 2^16 + 1/2) / 2^16.
__device__ __forceinline__ uint32_t random_m4(const float* x, const uint32_t* word) {
    int w = 0;
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[0], random_bits(word[0]), w, 0);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[1], random_bits(word[1]), w, 1);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[2], random_bits(word[2]), w, 2);
    return (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(x[3], random_bits(word[3]), w, 3);
}

// The same with the words' high halves and the probabilities that keep the mean of the square: cut off first, then one further
// where (x^2 - low^2) / (high^2 - low^2) is above the random number.  x is 0 or at least the least value.  Above the
// largest value there is NaN, which no comparison chooses.
__device__ __forceinline__ uint32_t random_r4(const float* x, const uint32_t* word) {
    int w = 0;
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[0], 0, w, 0);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[1], 0, w, 1);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[2], 0, w, 2);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(x[3], 0, w, 3);
    const int above = w + 0x01010101;
    const auto l01 = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), l23 = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    const auto h01 = __builtin_amdgcn_cvt_pk_f32_fp8(above, false), h23 = __builtin_amdgcn_cvt_pk_f32_fp8(above, true);
    const float low[4] = {l01[0], l01[1], l23[0], l23[1]}, high[4] = {h01[0], h01[1], h23[0], h23[1]};
    uint32_t out = (uint32_t)w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float u = fmaf((float)(word[k] >> 16), 0x1p-16f, 0x1p-17f);
        const bool up = (x[k] - low[k]) * (x[k] + low[k]) > (high[k] - low[k]) * u * (high[k] + low[k]);
        out += up ? 1u << (8 * k) : 0u;
    }
    return out;
}

// A wave's chunk: two blocks of a tensor, from the `at`-th element on, `n` elements of them.  Half of the wave takes a block,
// each lane four elements of its first half and four of its second, so that every access of the wave is to whole lines.
template <bool ONCE, typename P, typename G>
__device__ __forceinline__ void blocks_8(const StepArgs<true>& a, const Step8& s, int64_t at, int32_t n) {
    constexpr int V = 8, kApart = kStateBlock / 2;
    const int32_t lane = threadIdx.x % 64, begin = lane / 32 * kStateBlock, i = begin + lane % 32 * 4;
    const int64_t from = at + i, block = (at + begin) / kStateBlock;
    const bool there = begin < n, whole = i + kApart + 4 <= n;
    Raw<4, P> rp[2] = {};
    Raw<4, G> rg[2] = {};
    float p[V], g[V], m[V], r[V];
    uint32_t mw[2] = {}, rw[2] = {};
    uint8_t* const mq = (uint8_t*)s.m + from;
    uint8_t* const rq = (uint8_t*)s.v + from;
    P* const pp = (P*)s.p + from;
    const G* const pg = (const G*)s.g + from;
    if (whole) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            rp[j] = fetch_raw<4, ONCE>(pp + j * kApart);
            rg[j] = fetch_raw<4, ONCE>(pg + j * kApart);
            mw[j] = fetch_4<ONCE>(mq + j * kApart);
            rw[j] = fetch_4<ONCE>(rq + j * kApart);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int32_t e = k / 4 * kApart + k % 4;
            if (i + e < n) {
                rp[k / 4].t[k % 4] = pp[e];
                rg[k / 4].t[k % 4] = pg[e];
                mw[k / 4] |= (uint32_t)mq[e] << (8 * (k % 4));
                rw[k / 4] |= (uint32_t)rq[e] << (8 * (k % 4));
            }
        }
    }
    const float ms = there ? s.ms[block] : 0.0f, rs = there ? s.vs[block] : 0.0f;
    // Only now, with the elements on their way, what all of them share: 354 M weights take 912 us so and 932 with this first,
    // with step and learning rate on the GPU 955 and 1,002.  (States of 32 bits 1,546 with it first and 1,620 so.)
    const Common c = common_of(a);
    const float keep = (float)(1.0 - c.lr * (double)s.decay);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        p[k] = (float)rp[k / 4].t[k % 4];
        g[k] = (float)rg[k / 4].t[k % 4];
    }
#pragma unroll
    for (int k = 0; k < V / 4; ++k) {
        const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mw[k], false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mw[k], true);
        const auto r01 = __builtin_amdgcn_cvt_pk_f32_fp8(rw[k], false), r23 = __builtin_amdgcn_cvt_pk_f32_fp8(rw[k], true);
        m[4 * k] = m01[0], m[4 * k + 1] = m01[1], m[4 * k + 2] = m23[0], m[4 * k + 3] = m23[1];
        r[4 * k] = r01[0], r[4 * k + 1] = r01[1], r[4 * k + 2] = r23[0], r[4 * k + 3] = r23[1];
    }
    uint32_t least = 0xFFFFFFFFu;  // below the bits of v > 0
#pragma unroll
    for (int k = 0; k < V; ++k) {
        next_moments(c, g[k] * c.f, m[k] * ms, r[k] * rs, m[k], r[k]);
        least = min(least, __float_as_uint(r[k]) - 1);
    }
    if (least < __float_as_uint(kSmallRoot)) {
#pragma unroll
        for (int k = 0; k < V; ++k) r[k] = sqrtf(r[k]);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) r[k] = root(r[k]);
    }
    // The instruction takes a denormal number for 0, whose inverse makes NaN of an m of 0, and gives 0 instead of a denormal
    // one.  Without eps the sum is 0 or at least 2^-75, and r c.root stays below 2^91.
    if (c.eps == 0.0f || (c.eps >= 0x1p-126f && c.eps <= 0x1p100f)) {
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] = p[k] * keep - c.rate * m[k] * __builtin_amdgcn_rcpf(r[k] * c.root + c.eps);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] = p[k] * keep - c.rate * m[k] / (r[k] * c.root + c.eps);
    }
    if (whole) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float four[4] = {p[4 * j], p[4 * j + 1], p[4 * j + 2], p[4 * j + 3]};
            put_vec<ONCE>(pp + j * kApart, four);
            if (s.copy) store_copy<ONCE>(s.copy, s.ct, from + j * kApart, four);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int32_t e = k / 4 * kApart + k % 4;
            if (i + e < n) {
                const float one[1] = {p[k]};
                store_vec(pp + e, one);
                if (s.copy) store_copy<false>(s.copy, s.ct, from + e, one);
            }
        }
    }
    uint32_t most_m = 0, most_r = 0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        most_m = max(most_m, __float_as_uint(m[k]) & 0x7FFFFFFFu);
        most_r = max(most_r, __float_as_uint(r[k]));
    }
    most_m = block_most(most_m);
    most_r = block_most(most_r);
    uint32_t lost[V / 4] = {};
    if (__ballot(max(most_m, most_r) > kLargest)) {  // infinite values and NaN leave the others their scale
        most_m = most_r = 0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const uint32_t x = __float_as_uint(m[k]) & 0x7FFFFFFFu, y = __float_as_uint(r[k]);
            most_m = max(most_m, x <= kLargest ? x : 0u);
            most_r = max(most_r, y <= kLargest ? y : 0u);
            if (y > kLargest) lost[k / 4] |= 0x7Fu << (8 * (k % 4));
        }
        most_m = block_most(most_m);
        most_r = block_most(most_r);
    }
    const float to_m = e4m3_scale(__uint_as_float(most_m)), to_r = e4m3_scale(__uint_as_float(most_r));
    divide(m, to_m);
    divide(r, to_r);
    const uint32_t key = murmur_fmix32(c.key + (uint32_t)s.place) + (uint32_t)((uint64_t)at >> 32);
#pragma unroll
    for (int k = 0; k < V / 4; ++k) {
        uint32_t word[4];
#pragma unroll
        for (int l = 0; l < 4; ++l) {
            float& x = r[4 * k + l];
            word[l] = murmur_fmix32((uint32_t)(from + k * kApart + l) ^ key);
            x = x == 0.0f ? 0.0f : fmaxf(x, kLeast);  // of r > 0 no quotient is 0: from 2^-75 to 2^64 they differ by 2^139
        }
        mw[k] = random_m4(m + 4 * k, word);
        rw[k] = random_r4(r + 4 * k, word) | lost[k];
    }
    if (there && i == begin) {
        s.ms[block] = to_m;
        s.vs[block] = to_r;
    }
    if (whole) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            put_4<ONCE>(mq + j * kApart, mw[j]);
            put_4<ONCE>(rq + j * kApart, rw[j]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int32_t e = k / 4 * kApart + k % 4;
            if (i + e < n) {
                mq[e] = (uint8_t)(mw[k / 4] >> (8 * (k % 4)));
                rq[e] = (uint8_t)(rw[k / 4] >> (8 * (k % 4)));
            }
        }
    }
}

// EIGHT: the tensors of a launch have states in 8 bits.  ONCE: past the caches.
template <bool EIGHT, bool ONCE>
__global__ void __launch_bounds__(kStepThreads) k_adamw(StepArgs<EIGHT> a) {
    static_assert(kStepChunk8 == 2 * kStateBlock, "one turn");
    Common c;
    if constexpr (!EIGHT) c = common_of(a);
    uint32_t chunk = blockIdx.x;
    if constexpr (EIGHT) {
        constexpr uint32_t kTurn = kXcds * kTogether8;
        if (chunk < gridDim.x / kTurn * kTurn) {  // workgroup b runs on XCD b mod 8
            const uint32_t on = chunk / kXcds;
            chunk = on / kTogether8 * kTurn + chunk % kXcds * kTogether8 + on % kTogether8;
        }
    }
    chunk += a.from;
    const uint32_t k = tensor_of(a, chunk);
    const auto& s = a.s[k];
    const int64_t at = (int64_t)(chunk - a.first[k]) * (EIGHT ? kStepChunk8 : kStepChunk) - early<EIGHT>(s.m);
    const auto step = [&](auto p, auto g) {
        if constexpr (EIGHT)
            blocks_8<ONCE, decltype(p), decltype(g)>(a, s, at, (int32_t)min(kStepChunk8, s.n - at));
        else
            chunk_32<ONCE, decltype(p), decltype(g)>(c, s, at);
    };
    if (s.pt == SCD_F32)
        s.gt == SCD_F32 ? step(float{}, float{}) : s.gt == SCD_BF16 ? step(float{}, bf16{}) : step(float{}, f16{});
    else if (s.pt == SCD_BF16)
        s.gt == SCD_F32 ? step(bf16{}, float{}) : step(bf16{}, bf16{});
    else
        s.gt == SCD_F32 ? step(f16{}, float{}) : step(f16{}, f16{});
}

// Whether all arrays of a tensor have its whole chunks at the beginning of 64 bytes, the least that memory is written in: what
// a chunk's stores fill need not be read first.  (kStepLine is coarser, 256 bytes of a state and 128 of an array of 16 bits.)
template <bool EIGHT>
bool whole_lines(const scd_adamw_span_t& t) {
    const int64_t at = -(int64_t)early<EIGHT>(t.m), state = EIGHT ? 1 : 4;
    const auto place = [at](const void* p, int64_t bytes) { return (uint64_t)(uintptr_t)p + (uint64_t)(at * bytes); };
    return ((place(t.param, type_bytes(t.param_type)) | place(t.grad, type_bytes(t.grad_type)) | place(t.m, state) | place(t.v, state) |
             (t.copy ? place(t.copy, 2) : 0)) % 64) == 0;
}

// The launches for the tensors with states of one kind; with `once`, those past the caches and those through them.
template <bool EIGHT, bool ONCE>
void launch_steps(const scd_adamw_span_t* spans, int64_t count, const scd_adamw_t& o, bool once, hipStream_t stream) {
    StepArgs<EIGHT> a;
    a.seed = o.seed;
    a.lr_dev = o.lr_dev;
    a.step_dev = o.step_dev;
    a.norm_dev = o.norm_dev;
    a.lr = o.lr;
    a.log_b1 = std::log(o.beta1);
    a.log_b2 = std::log(o.beta2);
    a.b1 = (float)o.beta1;
    a.b2 = (float)o.beta2;
    a.a1 = (float)(1.0 - o.beta1);
    a.a2 = (float)(1.0 - o.beta2);
    a.eps = (float)o.eps;
    a.max_norm = o.max_norm;
    a.step = o.step;
    a.rate = (float)(o.lr / -std::expm1((double)o.step * a.log_b1));
    a.root = (float)(1.0 / std::sqrt(-std::expm1((double)o.step * a.log_b2)));
    for (int64_t i = 0; i < count;) {
        a.count = 0;
        a.chunks = 0;
        for (; i < count && a.count < a.kMost; ++i) {
            const scd_adamw_span_t& t = spans[i];
            if (t.n == 0 || (t.state_type == SCD_E4M3) != EIGHT || (once && whole_lines<EIGHT>(t)) != ONCE) continue;
            auto& s = a.s[a.count];
            s.p = t.param;
            s.g = t.grad;
            s.m = t.m;
            s.v = t.v;
            s.copy = t.copy;
            s.n = t.n;
            s.decay = t.weight_decay;
            s.pt = (uint8_t)t.param_type;
            s.gt = (uint8_t)t.grad_type;
            s.ct = (uint8_t)t.copy_type;
            if constexpr (EIGHT) {
                s.ms = t.m_scale;
                s.vs = t.v_scale;
                s.place = (uint64_t)i;
            }
            a.first[a.count++] = a.chunks;
            a.chunks += (uint32_t)ceil_div(t.n + early<EIGHT>(t.m), EIGHT ? kStepChunk8 : kStepChunk);
        }
        for (int64_t from = 0; from < a.chunks; from += kStepBlocks) {
            a.from = (uint32_t)from;
            const uint32_t blocks = (uint32_t)std::min<int64_t>(kStepBlocks, a.chunks - from);
            k_adamw<EIGHT, ONCE><<<blocks, kStepThreads, EIGHT ? 0 : kStepLds, stream>>>(a);
        }
    }
}

}  // namespace
}  // namespace feat
}  // namespace scd

using namespace scd::feat;

extern "C" int scd_adamw(const scd_adamw_span_t* spans, int64_t count, const scd_adamw_t* options, void* stream) {
    if (count < 0 || (count > 0 && !spans)) return fail(SCD_ERR_INVALID, "bad spans");
    if (!options) return fail(SCD_ERR_INVALID, "options is null");
    const scd_adamw_t& o = *options;
    if (!o.lr_dev && !(std::isfinite(o.lr) && o.lr >= 0.0)) return fail(SCD_ERR_INVALID, "lr must be >= 0");
    if (!(o.beta1 >= 0.0 && o.beta1 < 1.0 && o.beta2 >= 0.0 && o.beta2 < 1.0)) return fail(SCD_ERR_INVALID, "betas must be in [0, 1)");
    if (!(std::isfinite(o.eps) && o.eps >= 0.0)) return fail(SCD_ERR_INVALID, "eps must be >= 0");
    if (o.norm_dev && !(o.max_norm >= 0.0f)) return fail(SCD_ERR_INVALID, "max_norm must be >= 0");
    if (!o.step_dev && o.step < 1) return fail(SCD_ERR_INVALID, "step must be >= 1");
    int64_t total = 0, bytes = 0;
    for (int64_t i = 0; i < count; ++i) {
        const scd_adamw_span_t& t = spans[i];
        if (!type_bytes(t.param_type) || !type_bytes(t.grad_type) || (t.grad_type != t.param_type && t.grad_type != SCD_F32 && t.param_type != SCD_F32))
            return fail(SCD_ERR_UNSUPPORTED, "span %lld: float32 parameters, or bfloat16 or float16 ones with gradients of that type or float32", (long long)i);
        if (t.state_type != SCD_F32 && t.state_type != SCD_E4M3) return fail(SCD_ERR_UNSUPPORTED, "span %lld: states are float32 or of 8 bits (e4m3)", (long long)i);
        if (t.copy && (t.param_type != SCD_F32 || (t.copy_type != SCD_BF16 && t.copy_type != SCD_F16)))
            return fail(SCD_ERR_UNSUPPORTED, "span %lld: copies are bfloat16 or float16, of float32 parameters", (long long)i);
        if (!(std::isfinite(t.weight_decay) && t.weight_decay >= 0.0f)) return fail(SCD_ERR_INVALID, "span %lld: weight_decay must be >= 0", (long long)i);
        if (t.n < 0 || t.n > kStepMost - total || (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v || (t.state_type == SCD_E4M3 && (!t.m_scale || !t.v_scale)))))
            return fail(SCD_ERR_INVALID, "span %lld: bad size or null pointer", (long long)i);
        total += t.n;
        bytes += t.n * (2 * type_bytes(t.param_type) + type_bytes(t.grad_type) + (t.state_type == SCD_F32 ? 16 : 4) + (t.copy ? 2 : 0));
    }
    if (total == 0) return SCD_OK;
    const bool once = bytes >= kStepOnce;
    launch_steps<false, false>(spans, count, o, once, (hipStream_t)stream);
    launch_steps<true, false>(spans, count, o, once, (hipStream_t)stream);
    if (once) {
        launch_steps<false, true>(spans, count, o, once, (hipStream_t)stream);
        launch_steps<true, true>(spans, count, o, once, (hipStream_t)stream);
    }
    return launched("scd_adamw");
}

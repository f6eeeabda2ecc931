// scd_adamw.hip -- one AdamW step over many tensors, with states in 32 bits or in 8 (gfx950).
//
// g = f grad, f = max_norm / norm if norm > max_norm else 1;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;
// p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps);  copy = p rounded.
//
// Bound by memory: every tensor is read once and written once.  The tensors' addresses travel in the launch's arguments
// (up to kSteps a launch), so that a call copies nothing to the GPU; a tensor is cut into chunks, and each workgroup takes a
// run of consecutive chunks.  Launches do not depend on one another, and no element on another one but for the scales.
//
// In 8 bits (e4m3) a block of 256 elements has one scale for m and one for r = sqrt(v): the square root halves the range of
// exponents that v would need.  A wave takes a block, four elements a lane.  States are rounded up or down at random: to the
// nearest, v, which moves by a thousandth of itself in a step where half a step of its 8 bits is 6 to 12 %, would never move
// again.  m goes up with the probability that keeps its mean, r with the one that keeps the mean of r^2; r > 0 never
// becomes 0, where m over it would be without bound.  The random numbers are a hash of seed, step, tensor and element.
#include <algorithm>
#include <cmath>

#include "scd_device.h"
#include "scd_e4m3.h"
#include "scd_feat.h"

namespace scd {
namespace feat {
namespace {

constexpr int kStepThreads = 256;
constexpr int kSteps = 44;          // tensors a launch: the arguments stay below 4 KB
constexpr int kStepBlocks = 2048;   // workgroups of a launch at most
constexpr int kStateBlock = 256;    // elements that share a scale: a wave's
constexpr int64_t kStepChunk = 4096;

struct Step {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* ms;
    float* vs;
    void* copy;
    int64_t n;
    uint32_t first;  // number of chunks before this tensor's
    uint32_t place;  // in the call's list
    float decay;
    uint8_t pt, gt, ct, st;
};
struct StepArgs {
    Step s[kSteps];
    uint32_t count;
    uint32_t chunks;
    uint32_t chunk;  // elements of a chunk
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* norm_dev;
    double lr;
    double log_b1, log_b2;
    float b1, b2, a1, a2;  // a = 1 - b
    float eps, max_norm;
    int64_t step;
};
static_assert(sizeof(StepArgs) <= 4096, "kernel arguments");

// What all elements of a launch share.
struct Common {
    float f, b1, b2, a1, a2, eps;
    float rate;  // lr / (1 - b1^t)
    float root;  // 1 / sqrt(1 - b2^t)
    double lr;
    uint32_t key;
};

__device__ __forceinline__ Common common_of(const StepArgs& a) {
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
    const int64_t t = a.step_dev ? max(*a.step_dev, (int64_t)1) : a.step;
    c.lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    // 1 - b^t without cancellation
    c.rate = (float)(c.lr / -expm1((double)t * a.log_b1));
    c.root = (float)(1.0 / sqrt(-expm1((double)t * a.log_b2)));
    c.key = murmur_fmix32(a.seed ^ murmur_fmix32((uint32_t)t));
    return c;
}

// The tensor that holds a chunk.
__device__ __forceinline__ uint32_t tensor_of(const StepArgs& a, uint32_t chunk) {
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

__device__ __forceinline__ float moved(const Common& c, float keep, float p, float m, float v) {
    return p * keep - c.rate * m / (sqrtf(v) * c.root + c.eps);
}

template <int V>
__device__ __forceinline__ void store_copy(void* copy, int32_t type, int64_t i, const float (&p)[V]) {
    if (type == SCD_BF16)
        store_vec((bf16*)copy + i, p);
    else
        store_vec((f16*)copy + i, p);
}

// V elements from the i-th on, states in 32 bits.
template <int V, typename P, typename G>
__device__ __forceinline__ void step_32(const Common& c, const Step& s, float keep, int64_t i) {
    float p[V], g[V], m[V], v[V];
    load_vec((const P*)s.p + i, p);
    load_vec((const G*)s.g + i, g);
    load_vec((const float*)s.m + i, m);
    load_vec((const float*)s.v + i, v);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        g[k] *= c.f;
        m[k] = c.b1 * m[k] + c.a1 * g[k];
        v[k] = c.b2 * v[k] + c.a2 * (g[k] * g[k]);
        p[k] = moved(c, keep, p[k], m[k], v[k]);
    }
    store_vec((P*)s.p + i, p);
    store_vec((float*)s.m + i, m);
    store_vec((float*)s.v + i, v);
    if (s.copy) store_copy(s.copy, s.ct, i, p);
}

template <typename P, typename G>
__device__ __forceinline__ void chunk_32(const Common& c, const Step& s, int64_t at, int32_t n) {
    const float keep = (float)(1.0 - c.lr * (double)s.decay);
    for (int32_t i = threadIdx.x * 4; i < n; i += kStepThreads * 4) {
        if (i + 4 <= n) {
            step_32<4, P, G>(c, s, keep, at + i);
        } else {
            for (int32_t k = i; k < n; ++k) step_32<1, P, G>(c, s, keep, at + k);
        }
    }
}

constexpr float kFinite = 0x1.fffffep127f;

// A value x >= 0 between the neighbours low and high.
struct Between {
    float low, high;
};
__device__ __forceinline__ Between around(float x) {
    const bool small = x < kLeastNormal;  // there the distance of neighbours is that of the binade above
    const float shift = small ? kLeastNormal : 0.0f;
    const uint32_t low = __float_as_uint(x + shift) & 0xFFF00000u;
    return Between{__uint_as_float(low) - shift, __uint_as_float(low + 0x00100000u) - shift};
}

// u: uniform in (0, 1).  NaN and infinities come out as they are, and as NaN in 8 bits.
__device__ __forceinline__ float random_m(float x, float u) {
    const Between b = around(fabsf(x));
    return copysignf(fabsf(x) - b.low > u * (b.high - b.low) ? b.high : b.low, x);
}
__device__ __forceinline__ float random_r(float x, float u) {
    const Between b = around(x);
    const bool up = (x - b.low) * (x + b.low) > u * (b.high - b.low) * (b.high + b.low) || (b.low == 0.0f && x > 0.0f);
    return up ? b.high : b.low;
}

// The averages of a state in 8 bits.  Every product and sum rounds by itself, and scaled() below as a division does: a
// state that lies at the border between up and down goes the same way wherever these formulas are computed in 32 bits.
__device__ __forceinline__ void next_moments(const Common& c, float g, float m0, float r0, float& m, float& v) {
#pragma clang fp contract(off)
    m = c.b1 * m0 + c.a1 * g;
    v = c.b2 * (r0 * r0) + c.a2 * (g * g);
}

// x / scale, rounded once: the product with the (rounded) inverse is off by two units at most, and the remainder corrects it.
__device__ __forceinline__ float scaled(float x, float scale, float inverse) {
    const float q = x * inverse;
    return fmaf(fmaf(-q, scale, x), inverse, q);
}

// A block of a tensor, from the `at`-th element on, `n` of them: a wave.
template <typename P, typename G>
__device__ __forceinline__ void block_8(const Common& c, const Step& s, float keep, int64_t at, int32_t n) {
    constexpr int V = 4;
    const int32_t lane = threadIdx.x % 64, i = lane * V;
    const int64_t from = at + i, block = at / kStateBlock;
    const bool whole = i + V <= n;
    float p[V] = {}, g[V] = {};
    uint32_t mw = 0, vw = 0;
    const uint8_t* const mq = (const uint8_t*)s.m + from;
    const uint8_t* const vq = (const uint8_t*)s.v + from;
    if (whole) {
        load_vec((const P*)s.p + from, p);
        load_vec((const G*)s.g + from, g);
        __builtin_memcpy(&mw, mq, 4);
        __builtin_memcpy(&vw, vq, 4);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (i + k < n) {
                p[k] = (float)((const P*)s.p)[from + k];
                g[k] = (float)((const G*)s.g)[from + k];
                mw |= (uint32_t)mq[k] << (8 * k);
                vw |= (uint32_t)vq[k] << (8 * k);
            }
    }
    const float ms = s.ms[block], vs = s.vs[block];
    const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mw, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mw, true);
    const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8(vw, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(vw, true);
    float m[V] = {m01[0], m01[1], m23[0], m23[1]}, v[V] = {v01[0], v01[1], v23[0], v23[1]};
    float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        g[k] *= c.f;
        next_moments(c, g[k], m[k] * ms, v[k] * vs, m[k], v[k]);
        p[k] = moved(c, keep, p[k], m[k], v[k]);
        v[k] = sqrtf(v[k]);
        most_m = fmaxf(most_m, fabsf(m[k]));
        most_v = fmaxf(most_v, v[k]);
    }
    most_m = group_max<64>(most_m, 64);
    most_v = group_max<64>(most_v, 64);
    if (!(fmaxf(most_m, most_v) <= kFinite)) {  // rare: infinite ones leave the others their scale
        most_m = most_v = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            most_m = fmaxf(most_m, fabsf(m[k]) <= kFinite ? fabsf(m[k]) : 0.0f);
            most_v = fmaxf(most_v, v[k] <= kFinite ? v[k] : 0.0f);
        }
        most_m = group_max<64>(most_m, 64);
        most_v = group_max<64>(most_v, 64);
    }
    const float to_m = e4m3_scale(most_m), to_v = e4m3_scale(most_v);
    const float im = 1.0f / to_m, iv = 1.0f / to_v;
    const uint32_t key = murmur_fmix32(c.key + s.place) + (uint32_t)((uint64_t)at >> 32);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const uint32_t word = murmur_fmix32((uint32_t)(from + k) ^ key);
        m[k] = random_m(scaled(m[k], to_m, im), ((float)(word & 0xFFFFu) + 0.5f) * 0x1p-16f);
        v[k] = random_r(scaled(v[k], to_v, iv), ((float)(word >> 16) + 0.5f) * 0x1p-16f);
    }
    mw = e4m3_pack4(m[0], m[1], m[2], m[3]);
    vw = e4m3_pack4(v[0], v[1], v[2], v[3]);
    if (lane == 0) {
        s.ms[block] = to_m;
        s.vs[block] = to_v;
    }
    uint8_t* const mo = (uint8_t*)s.m + from;
    uint8_t* const vo = (uint8_t*)s.v + from;
    if (whole) {
        store_vec((P*)s.p + from, p);
        __builtin_memcpy(mo, &mw, 4);
        __builtin_memcpy(vo, &vw, 4);
        if (s.copy) store_copy(s.copy, s.ct, from, p);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (i + k < n) {
                ((P*)s.p)[from + k] = (P)p[k];
                mo[k] = (uint8_t)(mw >> (8 * k));
                vo[k] = (uint8_t)(vw >> (8 * k));
                if (s.copy) {
                    const float one[1] = {p[k]};
                    store_copy(s.copy, s.ct, from + k, one);
                }
            }
    }
}

template <typename P, typename G>
__device__ __forceinline__ void chunk_8(const Common& c, const Step& s, int64_t at, int32_t n) {
    const float keep = (float)(1.0 - c.lr * (double)s.decay);
    for (int32_t b = threadIdx.x / 64 * kStateBlock; b < n; b += kStepThreads / 64 * kStateBlock)
        block_8<P, G>(c, s, keep, at + b, min(kStateBlock, n - b));
}

template <typename P, typename G>
__device__ __forceinline__ void chunk_step(const Common& c, const Step& s, int64_t at, int32_t n) {
    if (s.st == SCD_F32)
        chunk_32<P, G>(c, s, at, n);
    else
        chunk_8<P, G>(c, s, at, n);
}

__global__ void __launch_bounds__(kStepThreads) k_adamw(StepArgs a) {
    const Common c = common_of(a);
    const uint32_t c0 = (uint32_t)((uint64_t)a.chunks * blockIdx.x / gridDim.x);
    const uint32_t c1 = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / gridDim.x);
    uint32_t k = tensor_of(a, c0);
    for (uint32_t chunk = c0; chunk < c1; ++chunk) {
        while (k + 1 < a.count && a.s[k + 1].first <= chunk) ++k;
        const Step& s = a.s[k];
        const int64_t at = (int64_t)(chunk - s.first) * a.chunk;
        const int32_t n = (int32_t)min((int64_t)a.chunk, s.n - at);
        if (s.pt == SCD_F32) {
            if (s.gt == SCD_F32)
                chunk_step<float, float>(c, s, at, n);
            else if (s.gt == SCD_BF16)
                chunk_step<float, bf16>(c, s, at, n);
            else
                chunk_step<float, f16>(c, s, at, n);
        } else if (s.pt == SCD_BF16) {
            if (s.gt == SCD_F32)
                chunk_step<bf16, float>(c, s, at, n);
            else
                chunk_step<bf16, bf16>(c, s, at, n);
        } else {
            if (s.gt == SCD_F32)
                chunk_step<f16, float>(c, s, at, n);
            else
                chunk_step<f16, f16>(c, s, at, n);
        }
    }
}

}  // namespace
}  // namespace feat
}  // namespace scd

using namespace scd::feat;

extern "C" int scd_adamw(const scd_adamw_span_t* spans, int64_t count, const scd_adamw_t* options, void* stream) {
    constexpr int64_t kMost = int64_t(1) << 42;  // elements of a call: chunk numbers stay below 2^32
    if (count < 0 || (count > 0 && !spans)) return fail(SCD_ERR_INVALID, "bad spans");
    if (!options) return fail(SCD_ERR_INVALID, "options is null");
    const scd_adamw_t& o = *options;
    if (!o.lr_dev && !(std::isfinite(o.lr) && o.lr >= 0.0)) return fail(SCD_ERR_INVALID, "lr must be >= 0");
    if (!(o.beta1 >= 0.0 && o.beta1 < 1.0 && o.beta2 >= 0.0 && o.beta2 < 1.0)) return fail(SCD_ERR_INVALID, "betas must be in [0, 1)");
    if (!(std::isfinite(o.eps) && o.eps >= 0.0)) return fail(SCD_ERR_INVALID, "eps must be >= 0");
    if (o.norm_dev && !(o.max_norm >= 0.0f)) return fail(SCD_ERR_INVALID, "max_norm must be >= 0");
    if (!o.step_dev && o.step < 1) return fail(SCD_ERR_INVALID, "step must be >= 1");
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        const scd_adamw_span_t& t = spans[i];
        if (!type_bytes(t.param_type) || !type_bytes(t.grad_type) || (t.grad_type != t.param_type && t.grad_type != SCD_F32 && t.param_type != SCD_F32))
            return fail(SCD_ERR_UNSUPPORTED, "span %lld: float32 parameters, or bfloat16 or float16 ones with gradients of that type or float32", (long long)i);
        if (t.state_type != SCD_F32 && t.state_type != SCD_E4M3) return fail(SCD_ERR_UNSUPPORTED, "span %lld: states are float32 or of 8 bits (e4m3)", (long long)i);
        if (t.copy && (t.param_type != SCD_F32 || (t.copy_type != SCD_BF16 && t.copy_type != SCD_F16)))
            return fail(SCD_ERR_UNSUPPORTED, "span %lld: copies are bfloat16 or float16, of float32 parameters", (long long)i);
        if (!(std::isfinite(t.weight_decay) && t.weight_decay >= 0.0f)) return fail(SCD_ERR_INVALID, "span %lld: weight_decay must be >= 0", (long long)i);
        if (t.n < 0 || t.n > kMost - total || (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v || (t.state_type == SCD_E4M3 && (!t.m_scale || !t.v_scale)))))
            return fail(SCD_ERR_INVALID, "span %lld: bad size or null pointer", (long long)i);
        total += t.n;
    }
    if (total == 0) return SCD_OK;
    StepArgs a;
    // Small chunks where whole ones would leave CUs idle.
    a.chunk = (uint32_t)(total < kStepChunk * kStepBlocks ? kStepChunk / 4 : kStepChunk);
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
    hipStream_t s = (hipStream_t)stream;
    for (int64_t i = 0; i < count;) {
        a.count = 0;
        a.chunks = 0;
        for (; i < count && a.count < kSteps; ++i) {
            const scd_adamw_span_t& t = spans[i];
            if (t.n == 0) continue;
            a.s[a.count++] = Step{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, a.chunks, (uint32_t)i, t.weight_decay, (uint8_t)t.param_type,
                                  (uint8_t)t.grad_type, (uint8_t)t.copy_type, (uint8_t)t.state_type};
            a.chunks += (uint32_t)ceil_div(t.n, (int64_t)a.chunk);
        }
        if (a.count) k_adamw<<<std::min<uint32_t>(kStepBlocks, a.chunks), kStepThreads, 0, s>>>(a);
    }
    return launched("scd_adamw");
}

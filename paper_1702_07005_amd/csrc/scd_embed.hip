// scd_embed.hip -- table lookup with scaling and its gradient by sorted tokens (gfx950).
//
// Lookup: out[t] = s E[tok[t]].  Gradient: dE[v] = s sum_{t: tok[t]=v} g[t].  Both only move data: the
// lookup reads the rows in use once and writes n rows; the gradient reads n rows and writes the whole table.
//
// The gradient sorts (token, position) pairs by token with a stable radix sort, so that the rows of one token
// are consecutive and in ascending position; every run of equal tokens is then summed in registers and its
// row written once.  Runs are cut where a group's share of the sorted list ends; the pieces of a cut run
// go through the workspace in 32 bits and are added in order.  No atomics: results are bit-identical from
// call to call.  The zeros of the rows without a token are written while the sort, which moves
// little data, runs.
#include <algorithm>
#include <type_traits>

#include "scd_feat.h"

namespace scd {
namespace feat {
namespace {

constexpr int kThreads = 256;

// A row is `lanes` consecutive threads (a power of two, at most 256) with VEC elements each, and as many
// such column ranges (blockIdx.y) as it needs.  Rows narrower than 16 bytes go element by element (VEC = 1).
struct RowMap {
    uint32_t log2_lanes;
    uint32_t ranges;
};

RowMap row_map(int64_t dim, int vec) {
    RowMap m;
    m.log2_lanes = std::min<uint32_t>(8, log2_up((uint64_t)ceil_div(dim, vec)));
    m.ranges = (uint32_t)ceil_div(dim, (int64_t)vec << m.log2_lanes);
    return m;
}

// ---------------------------------------------------------------------------------------- lookup

template <int VEC, int U, typename TI, typename TT, typename TO>
__global__ void __launch_bounds__(kThreads) k_embed(const TI* __restrict__ tok, int64_t n, const TT* __restrict__ table,
                                                    int64_t tstride, int64_t rows, int32_t dim, float scale,
                                                    TO* __restrict__ out, int64_t ostride, uint32_t log2_lanes) {
    const int64_t groups = (int64_t)gridDim.x * (kThreads >> log2_lanes);
    const int64_t g = (int64_t)blockIdx.x * (kThreads >> log2_lanes) + (threadIdx.x >> log2_lanes);
    const int32_t k = (int32_t)((blockIdx.y << log2_lanes) + (threadIdx.x & ((1u << log2_lanes) - 1)));
    if (k * VEC >= dim) return;
    int32_t again;
    const int32_t c = vec_column<VEC>(k, dim, again);
    int64_t id[U];
    Raw<VEC, TT> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = g + u * groups < n ? (int64_t)tok[g + u * groups] : -1;
    if (rows > 0) {  // a token without a row reads row 0, so that the loads do not wait for one another's conditions
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_raw<VEC>(table + (id[u] >= 0 && id[u] < rows ? id[u] : 0) * tstride + c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float o[VEC];
        widen(v[u], o);
        const bool in = id[u] >= 0 && id[u] < rows;
        const float other = id[u] < 0 ? 0.0f : __builtin_nanf("");
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = in ? scale * o[i] : other;
        if (g + u * groups < n) store_vec(out + (g + u * groups) * ostride + c, o);
    }
}

// ---------------------------------------------------------------------------------------- sort
// Keys are the tokens; one outside [0, rows) gets the key `rows` and so comes last.  The list is padded to a whole
// number of batches of k_sums with such keys, at position 0.

constexpr int kBatch = 8;

template <typename TI>
struct Tokens {
    const TI* tok;
    int64_t n;
    uint32_t rows;
    __device__ uint32_t key(int64_t i) const {
        const int64_t t = i < n ? (int64_t)tok[i] : -1;
        return t >= 0 && t < (int64_t)rows ? (uint32_t)t : rows;
    }
    __device__ uint32_t pos(int64_t i) const { return i < n ? (uint32_t)i : 0; }
};
struct Pairs {
    const uint32_t* k;
    const uint32_t* p;
    __device__ uint32_t key(int64_t i) const { return k[i]; }
    __device__ uint32_t pos(int64_t i) const { return p[i]; }
};

// Fills this worker's share of the table's bytes with zeros.
struct Fill {
    char* p;            // null: nothing to fill
    int64_t rows;       // matrix of `rows` rows of row_bytes, `stride` bytes apart
    int64_t row_bytes;
    int64_t stride;
};

__device__ __forceinline__ void fill_bytes(char* p, int64_t bytes, int64_t worker, int64_t workers) {
    // 16-byte stores from the first aligned address on; what is left at both ends goes in 2-byte stores.
    const int64_t head = min(bytes, (int64_t)((16 - ((uintptr_t)p & 15)) & 15));
    const int64_t n16 = (bytes - head) / 16, tail = head + n16 * 16;
    uint4* q = reinterpret_cast<uint4*>(p + head);
    for (int64_t i = worker; i < n16; i += workers) q[i] = make_uint4(0, 0, 0, 0);
    for (int64_t i = worker * 2; i < head; i += workers * 2) *reinterpret_cast<uint16_t*>(p + i) = 0;
    for (int64_t i = tail + worker * 2; i < bytes; i += workers * 2) *reinterpret_cast<uint16_t*>(p + i) = 0;
}

__device__ __forceinline__ void fill_zero(const Fill& f, uint32_t block, uint32_t blocks) {
    if (f.stride == f.row_bytes) {
        fill_bytes(f.p, f.rows * f.row_bytes, (int64_t)block * blockDim.x + threadIdx.x, (int64_t)blocks * blockDim.x);
        return;
    }
    const int64_t waves = (int64_t)blocks * (blockDim.x / 64);
    for (int64_t r = (int64_t)block * (blockDim.x / 64) + threadIdx.x / 64; r < f.rows; r += waves)
        fill_bytes(f.p + r * f.stride, f.row_bytes, threadIdx.x % 64, 64);
}

// The lanes of the wave that hold the same digit as this one, among the active ones.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits) {
    uint64_t m = __ballot(1);
    for (int b = 0; b < bits; ++b) {
        const bool on = (digit >> b) & 1;
        const uint64_t v = __ballot(on);
        m &= on ? v : ~v;
    }
    return m;
}

__device__ __forceinline__ uint32_t lanes_below(uint64_t m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// Exclusive prefix sums over the threads of a workgroup of at most 1,024; `total` is the whole sum.
__device__ __forceinline__ uint32_t block_exclusive(uint32_t x, uint32_t* wave_sums, uint32_t& total) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    uint32_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(s, o);
        if (lane >= (uint32_t)o) s += y;
    }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
    for (uint32_t w = 0; w < waves; ++w) {
        const uint32_t t = wave_sums[w];
        before += w < wave ? t : 0;
        total += t;
    }
    __syncthreads();
    return before + s - x;
}

// Ranks the J x 64 consecutive keys of this wave among its own of the same digit; counts[digit] (the wave's,
// zeroed) becomes the wave's number of keys with that digit.
template <int J>
__device__ __forceinline__ void wave_ranks(const uint32_t (&digit)[J], const bool (&on)[J], int bits,
                                           volatile uint16_t* counts, uint32_t (&rank)[J]) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (!on[j]) continue;
        const uint64_t m = same_digit(digit[j], bits);
        const uint32_t below = lanes_below(m);
        const uint32_t base = counts[digit[j]];
        rank[j] = base + below;
        __builtin_amdgcn_wave_barrier();
        if (below == 0) counts[digit[j]] = (uint16_t)(base + (uint32_t)__popcll(m));
        __builtin_amdgcn_wave_barrier();
    }
}

// One workgroup sorts everything (n, the padded length, is at most 1,024 J): keys and positions stay in registers, each pass exchanges them
// through LDS.  The launch's other workgroups fill zeros.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;

template <int J>
constexpr size_t sort_one_lds(int bins) {
    return (size_t)kSortThreads * J * 6 + (size_t)kSortWaves * bins * 2 + 64 * 4;
}

template <int J, typename TI>
__global__ void __launch_bounds__(kSortThreads) k_sort_one(Tokens<TI> src, uint32_t n, int passes, int bits, uint32_t* __restrict__ keys,
                                                           uint32_t* __restrict__ pos, Fill fill) {
    if (blockIdx.x) {
        fill_zero(fill, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    extern __shared__ __align__(16) char lds[];
    const int bins = 1 << bits;
    uint32_t* const lkey = reinterpret_cast<uint32_t*>(lds);
    uint16_t* const lpos = reinterpret_cast<uint16_t*>(lkey + kSortThreads * J);
    uint16_t* const counts = lpos + kSortThreads * J;  // [waves][bins]
    uint32_t* const sums = reinterpret_cast<uint32_t*>(counts + kSortWaves * bins);
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, at = wave * 64 * J + lane;
    uint32_t key[J], place[J], digit[J], rank[J];
    bool on[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t i = at + j * 64;
        on[j] = i < n;
        key[j] = src.key(i);
        place[j] = src.pos(i);
    }
    for (int p = 0; p < passes; ++p) {
        for (int i = threadIdx.x; i < kSortWaves * bins / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(counts)[i] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < J; ++j) digit[j] = (key[j] >> (p * bits)) & (uint32_t)(bins - 1);
        wave_ranks<J>(digit, on, bits, counts + wave * bins, rank);
        __syncthreads();
        // Digit-major, wave-minor prefix sums of the counts (bins <= the threads).
        uint32_t c[kSortWaves], sum = 0, total;
        const bool mine = threadIdx.x < (uint32_t)bins;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            c[w] = mine ? counts[w * bins + threadIdx.x] : 0;
            sum += c[w];
        }
        uint32_t base = block_exclusive(sum, sums, total);
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            if (mine) counts[w * bins + threadIdx.x] = (uint16_t)base;
            base += c[w];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (on[j]) {
                const uint32_t to = counts[wave * bins + digit[j]] + rank[j];
                lkey[to] = key[j];
                lpos[to] = (uint16_t)place[j];
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < J; ++j) {
            key[j] = lkey[at + j * 64];
            place[j] = lpos[at + j * 64];
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (on[j]) {
            keys[at + j * 64] = key[j];
            pos[at + j * 64] = place[j];
        }
}

// Many workgroups: a tile of kTile consecutive keys each; per pass the tiles' digit counts (k_sort_count),
// their prefix sums along each digit (k_sort_scan), and the move (k_sort_move).  Each launch fills a part of the
// zeros with extra workgroups.
constexpr int kTileThreads = 512;
constexpr int kTileJ = 8;
constexpr int kTile = kTileThreads * kTileJ;
constexpr int kMaxBits = 11;

template <typename SRC>
__global__ void __launch_bounds__(kTileThreads) k_sort_count(SRC src, int64_t n, int shift, int bits, uint32_t tiles,
                                                             uint32_t* __restrict__ hist, Fill fill) {
    if (blockIdx.x >= tiles) {
        fill_zero(fill, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    __shared__ uint32_t count[1 << kMaxBits];
    const int bins = 1 << bits;
    for (int i = threadIdx.x; i < bins; i += kTileThreads) count[i] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kTile;
#pragma unroll
    for (int j = 0; j < kTileJ; ++j) {
        const int64_t i = base + j * kTileThreads + threadIdx.x;
        if (i < n) atomicAdd(&count[(src.key(i) >> shift) & (uint32_t)(bins - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += kTileThreads) hist[(int64_t)i * tiles + blockIdx.x] = count[i];
}

// One wave per digit: hist[digit][tile] becomes the digit's count in the tiles before, totals[digit] in all.
__global__ void __launch_bounds__(kThreads) k_sort_scan(uint32_t* __restrict__ hist, uint32_t tiles, uint32_t bins,
                                                        uint32_t* __restrict__ totals, Fill fill) {
    const uint32_t scans = (bins + kThreads / 64 - 1) / (kThreads / 64);
    if (blockIdx.x >= scans) {
        fill_zero(fill, blockIdx.x - scans, gridDim.x - scans);
        return;
    }
    const uint32_t lane = threadIdx.x % 64, d = blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (d >= bins) return;
    uint32_t* const h = hist + (int64_t)d * tiles;
    uint32_t before = 0;
    for (uint32_t t = 0; t < tiles; t += 64) {
        const uint32_t x = t + lane < tiles ? h[t + lane] : 0;
        uint32_t s = x;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = __shfl_up(s, o);
            if (lane >= (uint32_t)o) s += y;
        }
        if (t + lane < tiles) h[t + lane] = before + s - x;
        before += __shfl(s, 63);
    }
    if (lane == 0) totals[d] = before;
}

template <typename SRC>
__global__ void __launch_bounds__(kTileThreads) k_sort_move(SRC src, int64_t n, int shift, int bits, uint32_t tiles,
                                                            const uint32_t* __restrict__ hist,
                                                            const uint32_t* __restrict__ totals,
                                                            uint32_t* __restrict__ keys, uint32_t* __restrict__ pos, Fill fill) {
    if (blockIdx.x >= tiles) {
        fill_zero(fill, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    constexpr int kWaves = kTileThreads / 64;
    constexpr int kPer = (1 << kMaxBits) / kTileThreads;
    __shared__ uint16_t counts[kWaves << kMaxBits];
    __shared__ uint32_t start[1 << kMaxBits];
    __shared__ uint32_t sums[kWaves];
    const int bins = 1 << bits;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int i = threadIdx.x; i < kWaves * bins; i += kTileThreads) counts[i] = 0;
    // Where each digit's keys of this tile begin: the smaller digits' totals and the tiles before.
    uint32_t t[kPer], sum = 0, total;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int d = (int)threadIdx.x * kPer + k;
        t[k] = d < bins ? totals[d] : 0;
        sum += t[k];
    }
    uint32_t base = block_exclusive(sum, sums, total);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int d = (int)threadIdx.x * kPer + k;
        if (d < bins) start[d] = base + hist[(int64_t)d * tiles + blockIdx.x];
        base += t[k];
    }
    const int64_t at = (int64_t)blockIdx.x * kTile + wave * 64 * kTileJ + lane;
    uint32_t key[kTileJ], place[kTileJ], digit[kTileJ], rank[kTileJ];
    bool on[kTileJ];
#pragma unroll
    for (int j = 0; j < kTileJ; ++j) {
        const int64_t i = at + j * 64;
        on[j] = i < n;
        key[j] = on[j] ? src.key(i) : 0;
        place[j] = on[j] ? src.pos(i) : 0;
        digit[j] = (key[j] >> shift) & (uint32_t)(bins - 1);
    }
    __syncthreads();
    wave_ranks<kTileJ>(digit, on, bits, counts + wave * bins, rank);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kTileThreads) {
        uint32_t b = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = counts[w * bins + d];
            counts[w * bins + d] = (uint16_t)b;
            b += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kTileJ; ++j)
        if (on[j]) {
            const uint32_t to = start[digit[j]] + counts[wave * bins + digit[j]] + rank[j];
            keys[to] = key[j];
            pos[to] = place[j];
        }
}

// ---------------------------------------------------------------------------------------- sums
// Group g sums entries [g S, (g+1) S) of the sorted list, run by run.  A run that lies inside is final.  Of a cut
// run, the group where it ends keeps its piece in head[g], the groups before theirs in tail[g]; k_sums_join adds
// them in order.  All pieces are 32 bits and unscaled.

struct SumArgs {
    const uint32_t* keys;
    const uint32_t* pos;
    int64_t n;
    uint32_t share;  // S
    uint32_t rows;
    int32_t dim;
    float scale;
    int64_t gstride, ostride;
    float* head;  // [groups][dim]
    float* tail;
};

// `again` columns of the vector belong to the vector before: they may be written twice, but added to once.
template <int VEC, bool ACC, typename TO>
__device__ __forceinline__ void write_row(const SumArgs& a, TO* __restrict__ out, uint32_t row, int32_t c, int32_t again,
                                          const float (&s)[VEC]) {
    float v[VEC];
    TO* const p = out + (int64_t)row * a.ostride + c;
    if constexpr (ACC) {
        load_vec(p, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] += a.scale * s[i];
        if (again) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i >= again) p[i] = (TO)v[i];
            return;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = a.scale * s[i];
    }
    store_vec(p, v);
}

template <int VEC, bool ACC, typename TG, typename TO>
__global__ void __launch_bounds__(kThreads) k_sums(SumArgs a, const TG* __restrict__ grad, TO* __restrict__ out, uint32_t log2_lanes) {
    constexpr int U = kBatch;  // divides the share and the list
    const int64_t g = (int64_t)blockIdx.x * (kThreads >> log2_lanes) + (threadIdx.x >> log2_lanes);
    const int32_t col = (int32_t)((blockIdx.y << log2_lanes) + (threadIdx.x & ((1u << log2_lanes) - 1)));
    const int64_t e0 = g * a.share, e1 = min(a.n, e0 + a.share);
    if (e0 >= a.n || col * VEC >= a.dim) return;
    int32_t again;
    const int32_t c = vec_column<VEC>(col, a.dim, again);
    uint32_t cur = a.keys[e0];
    bool cut = e0 > 0 && a.keys[e0 - 1] == cur;
    float acc[VEC] = {};
    for (int64_t e = e0; e < e1; e += U) {
        const Raw<U, uint32_t> k = load_raw<U>(a.keys + e), p = load_raw<U>(a.pos + e);
        Raw<VEC, TG> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            v[u] = load_raw<VEC>(grad + (int64_t)p.t[u] * a.gstride + c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k.t[u] != cur) {
                if (cut)
                    store_vec(a.head + g * a.dim + c, acc);
                else
                    write_row<VEC, ACC>(a, out, cur, c, again, acc);
                cut = false;
                cur = k.t[u];
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
            }
            float x[VEC];
            widen(v[u], x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += x[i];
        }
    }
    if (cur >= a.rows) return;
    if (e1 < a.n && a.keys[e1] == cur)
        store_vec(a.tail + g * a.dim + c, acc);
    else if (cut)
        store_vec(a.head + g * a.dim + c, acc);
    else
        write_row<VEC, ACC>(a, out, cur, c, again, acc);
}

// The sum of tail[first], tail[first + step], ... below `end`, for the vector at column c.
template <int VEC>
__device__ __forceinline__ void add_tails(const SumArgs& a, int64_t first, int64_t end, int64_t step, int32_t c, float (&s)[VEC]) {
    constexpr int U = 8;
    for (int64_t g = first; g < end; g += U * step) {
        Raw<VEC, float> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            v[u] = load_raw<VEC>(a.tail + (g + u * step < end ? g + u * step : g) * a.dim + c);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[i] += g + u * step < end ? v[u].t[i] : 0.0f;
    }
}

// The group (at most g) in which the run that ends in group g begins.
__device__ __forceinline__ int64_t run_begins(const SumArgs& a, int64_t g, uint32_t row) {
    int64_t lo = 0, hi = g * a.share;  // keys[hi] == row
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (a.keys[mid] < row)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo / a.share;
}

// Rows cut into at most kShortRun pieces are joined by their group; longer ones then by the whole workgroup, group j
// taking every m-th piece from the j-th on and the m sums added in order.
constexpr int kShortRun = 16;

template <int VEC, bool ACC, typename TO>
__global__ void __launch_bounds__(kThreads) k_sums_join(SumArgs a, TO* __restrict__ out, uint32_t log2_lanes) {
    __shared__ float part[kThreads * VEC];
    __shared__ int64_t ends[kThreads], begins[kThreads];
    const uint32_t m = kThreads >> log2_lanes, j = threadIdx.x >> log2_lanes, l = threadIdx.x & ((1u << log2_lanes) - 1);
    const int64_t g = (int64_t)blockIdx.x * m + j;
    const int32_t col = (int32_t)((blockIdx.y << log2_lanes) + l);
    const bool in = col * VEC < a.dim;
    int32_t again;
    const int32_t c = vec_column<VEC>(in ? col : 0, a.dim, again);
    const int64_t e0 = g * a.share, e1 = min(a.n, e0 + a.share);
    int64_t begin = -1;
    uint32_t row = 0;
    if (e0 > 0 && e0 < a.n) {
        row = a.keys[e0];
        if (row < a.rows && a.keys[e0 - 1] == row && (e1 == a.n || a.keys[e1] != row)) begin = run_begins(a, g, row);
    }
    const bool is_long = begin >= 0 && g - begin > kShortRun;
    if (l == 0) {
        ends[j] = is_long ? g : -1;
        begins[j] = begin;
    }
    if (begin >= 0 && !is_long && in) {
        float s[VEC] = {}, h[VEC];
        add_tails<VEC>(a, begin, g, 1, c, s);
        load_vec(a.head + g * a.dim + c, h);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] += h[i];
        write_row<VEC, ACC>(a, out, row, c, again, s);
    }
    __syncthreads();
    for (uint32_t q = 0; q < m; ++q) {
        const int64_t end = ends[q];
        if (end < 0) continue;
        float s[VEC] = {};
        if (in) add_tails<VEC>(a, begins[q] + j, end, m, c, s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[threadIdx.x * VEC + i] = s[i];
        __syncthreads();
        if (j == 0 && in) {
            for (uint32_t k = 1; k < m; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[i] += part[((k << log2_lanes) + l) * VEC + i];
            float h[VEC];
            load_vec(a.head + end * a.dim + c, h);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[i] += h[i];
            write_row<VEC, ACC>(a, out, a.keys[end * a.share], c, again, s);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------- host

// Elements per thread and row: 16 bytes of the wider of the two types; 1 where a row has fewer.
int vec_for(int32_t a, int32_t b, int64_t dim) {
    const int vec = 16 / std::max(type_bytes(a), type_bytes(b));
    return dim < vec ? 1 : vec;
}

// Calls f(A{}, B{}, Int<vec_for(a, b, dim)>{}).
template <typename F>
void with_vec(int32_t a, int32_t b, int64_t dim, F&& f) {
    with_type(a, [&](auto ta) {
        with_type(b, [&](auto tb) {
            constexpr int VEC = 16 / (sizeof(ta) > sizeof(tb) ? sizeof(ta) : sizeof(tb));
            dim < VEC ? f(ta, tb, Int<1>{}) : f(ta, tb, Int<VEC>{});
        });
    });
}

bool is_element(int32_t t) { return type_bytes(t) != 0; }
bool is_token(int32_t t) { return t == SCD_I32 || t == SCD_I64; }

// How a gradient call sorts and splits: a function of the sizes alone.
struct Plan {
    int64_t n;        // padded to whole batches
    bool one;         // one workgroup sorts
    int passes, bits;
    int64_t tiles;
    uint32_t share;
    int64_t groups;
    int64_t pairs;    // bytes of one key or position array
    int64_t hist, pieces, bytes;
};

constexpr int64_t kSortOneMax = int64_t(kSortThreads) * 16;

int64_t align16(int64_t b) { return (b + 15) / 16 * 16; }

Plan plan_for(int64_t n, int64_t rows, int64_t dim) {
    Plan p{};
    p.n = ceil_div(n, kBatch) * kBatch;
    p.one = p.n <= kSortOneMax;
    const int key_bits = (int)log2_up((uint64_t)rows + 1);
    const int most = p.one ? 9 : kMaxBits;
    p.passes = std::max(1, (key_bits + most - 1) / most);
    p.bits = std::max(1, (key_bits + p.passes - 1) / p.passes);
    p.tiles = p.one ? 0 : ceil_div(p.n, kTile);
    // Entries per group: as many as keep about 4,096 waves in work, 8 at least, 64 at most.
    const int64_t work = p.n * ceil_div(dim, 4) / 64;
    p.share = (uint32_t)std::min<int64_t>(64, std::max<int64_t>(8, work / 4096 / 8 * 8));
    p.groups = ceil_div(p.n, p.share);
    p.pairs = p.n * 4;
    p.hist = p.one ? 0 : align16(((p.tiles + 1) << p.bits) * 4);
    p.pieces = align16(p.groups * dim * 4);
    p.bytes = (p.one ? 2 : 4) * p.pairs + p.hist + 2 * p.pieces;
    return p;
}

// Workgroups of `threads` threads that fill a part of the zeros beside other work: 64 KB each, at most as many as the
// GPU has CUs (a few each where the others are small).
uint32_t fill_blocks(const Fill& f, int threads) {
    if (!f.p) return 0;
    return (uint32_t)std::min<int64_t>(ceil_div(f.rows * f.row_bytes, 65536), 255 * (1024 / threads));
}

template <int J, typename TI>
int launch_sort_one(Tokens<TI> src, const Plan& p, uint32_t* keys, uint32_t* pos, const Fill& fill, hipStream_t s) {
    const size_t lds = sort_one_lds<J>(1 << p.bits);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_sort_one<J, TI>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return fail(SCD_ERR_HIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
    k_sort_one<J, TI><<<1 + fill_blocks(fill, kSortThreads), kSortThreads, lds, s>>>(src, (uint32_t)p.n, p.passes, p.bits, keys, pos, fill);
    return launched("sort of tokens");
}

template <typename SRC>
void launch_pass(SRC src, int pass, const Plan& p, uint32_t* hist, uint32_t* totals, uint32_t* keys, uint32_t* pos, Fill* fills, hipStream_t s) {
    const uint32_t tiles = (uint32_t)p.tiles, bins = 1u << p.bits;
    k_sort_count<<<tiles + fill_blocks(fills[0], kTileThreads), kTileThreads, 0, s>>>(src, p.n, pass * p.bits, p.bits, tiles, hist, fills[0]);
    k_sort_scan<<<(uint32_t)ceil_div(bins, kThreads / 64) + fill_blocks(fills[1], kThreads), kThreads, 0, s>>>(hist, tiles, bins, totals, fills[1]);
    k_sort_move<<<tiles + fill_blocks(fills[2], kTileThreads), kTileThreads, 0, s>>>(src, p.n, pass * p.bits, p.bits, tiles, hist, totals, keys, pos, fills[2]);
}

}  // namespace
}  // namespace feat
}  // namespace scd

using namespace scd::feat;

extern "C" int scd_embed(const void* tokens, int32_t token_type, int64_t n, const void* table, int32_t table_type,
                         int64_t table_stride, int64_t rows, int64_t dim, float scale, void* out, int32_t out_type,
                         int64_t out_stride, void* stream) {
    if (!is_token(token_type) || !is_element(table_type) || !is_element(out_type))
        return fail(SCD_ERR_UNSUPPORTED, "scd_embed takes int32 or int64 tokens and float32, bfloat16 or float16 rows");
    if (n < 0 || n > kMaxRows || rows < 0 || rows > kMaxRows || dim < 1 || dim > kMaxDim)
        return fail(SCD_ERR_INVALID, "bad sizes n=%lld rows=%lld dim=%lld", (long long)n, (long long)rows, (long long)dim);
    if (table_stride < 0 || (out_stride < dim && n > 1)) return fail(SCD_ERR_INVALID, "bad row stride");
    if (n == 0) return SCD_OK;
    if (!tokens || (!table && rows > 0) || !out) return fail(SCD_ERR_INVALID, "null device pointer");
    const int vec = vec_for(table_type, out_type, dim);
    const RowMap m = row_map(dim, vec);
    const int64_t per = kThreads >> m.log2_lanes;
    // Four rows per thread in flight once that still leaves eight workgroups to each CU.
    const int U = ceil_div(n, per * 4) * m.ranges >= 2048 ? 4 : 1;
    const dim3 grid((uint32_t)ceil_div(n, per * U), m.ranges);
    with_vec(table_type, out_type, dim, [&](auto tt, auto to, auto vc) {
        using TT = decltype(tt);
        using TO = decltype(to);
        constexpr int VEC = decltype(vc)::value;
        const auto go = [&](auto ti, auto uc) {
            using TI = decltype(ti);
            constexpr int U = decltype(uc)::value;
            k_embed<VEC, U><<<grid, kThreads, 0, (hipStream_t)stream>>>((const TI*)tokens, n, (const TT*)table, table_stride, rows,
                                                                       (int32_t)dim, scale, (TO*)out, out_stride, m.log2_lanes);
        };
        if (token_type == SCD_I32)
            U == 4 ? go(int32_t{}, Int<4>{}) : go(int32_t{}, Int<1>{});
        else
            U == 4 ? go(int64_t{}, Int<4>{}) : go(int64_t{}, Int<1>{});
    });
    return launched("scd_embed");
}

extern "C" int scd_embed_grad_workspace(int64_t n, int64_t rows, int64_t dim, int64_t* bytes) {
    if (!bytes) return fail(SCD_ERR_INVALID, "bytes is null");
    *bytes = 0;
    if (n < 0 || n > kMaxRows || rows < 0 || rows > kMaxRows || dim < 1 || dim > kMaxDim)
        return fail(SCD_ERR_INVALID, "bad sizes n=%lld rows=%lld dim=%lld", (long long)n, (long long)rows, (long long)dim);
    if (n > 0 && rows > 0) *bytes = plan_for(n, rows, dim).bytes;
    return SCD_OK;
}

extern "C" int scd_embed_grad(const void* tokens, int32_t token_type, int64_t n, const void* grad, int32_t grad_type,
                              int64_t grad_stride, int64_t rows, int64_t dim, float scale, int32_t accumulate, void* out,
                              int32_t out_type, int64_t out_stride, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!is_token(token_type) || !is_element(grad_type) || !is_element(out_type))
        return fail(SCD_ERR_UNSUPPORTED, "scd_embed_grad takes int32 or int64 tokens and float32, bfloat16 or float16 rows");
    if (n < 0 || n > kMaxRows || rows < 0 || rows > kMaxRows || dim < 1 || dim > kMaxDim)
        return fail(SCD_ERR_INVALID, "bad sizes n=%lld rows=%lld dim=%lld", (long long)n, (long long)rows, (long long)dim);
    if (grad_stride < 0 || (out_stride < dim && rows > 1)) return fail(SCD_ERR_INVALID, "bad row stride");
    if (rows == 0 || (n == 0 && accumulate)) return SCD_OK;
    if (!out || (n > 0 && (!tokens || !grad))) return fail(SCD_ERR_INVALID, "null device pointer");
    hipStream_t s = (hipStream_t)stream;
    const int64_t e = type_bytes(out_type);
    Fill fill{};
    if (!accumulate) fill = Fill{(char*)out, rows, dim * e, rows > 1 ? out_stride * e : dim * e};
    const Plan p = plan_for(n, rows, dim);
    if (n > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < p.bytes))
        return fail(SCD_ERR_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)p.bytes);
    char* w = (char*)workspace;
    uint32_t* keys = (uint32_t*)w;
    uint32_t* pos = (uint32_t*)(w + p.pairs);
    int rc = SCD_OK;
    const auto sort = [&](auto ti) {
        using TI = decltype(ti);
        const Tokens<TI> src{(const TI*)tokens, n, (uint32_t)rows};
        if (p.one) {
            if (p.n <= kSortThreads)
                rc = launch_sort_one<1>(src, p, keys, pos, fill, s);
            else if (p.n <= 4 * kSortThreads)
                rc = launch_sort_one<4>(src, p, keys, pos, fill, s);
            else
                rc = launch_sort_one<16>(src, p, keys, pos, fill, s);
            return;
        }
        // The passes' launches share the zeros evenly.
        uint32_t* const other_keys = (uint32_t*)(w + 2 * p.pairs);
        uint32_t* const other_pos = (uint32_t*)(w + 3 * p.pairs);
        uint32_t* const hist = (uint32_t*)(w + 4 * p.pairs);
        uint32_t* const totals = hist + (p.tiles << p.bits);
        const int launches = 3 * p.passes;
        for (int k = 0; k < p.passes; ++k) {
            Fill part[3] = {};
            for (int j = 0; fill.p && j < 3; ++j) {
                const int64_t a = rows * (3 * k + j) / launches, b = rows * (3 * k + j + 1) / launches;
                if (b > a) part[j] = Fill{fill.p + a * fill.stride, b - a, fill.row_bytes, fill.stride};
            }
            uint32_t* const to_keys = k % 2 ? other_keys : keys;
            uint32_t* const to_pos = k % 2 ? other_pos : pos;
            if (k == 0)
                launch_pass(src, k, p, hist, totals, to_keys, to_pos, part, s);
            else
                launch_pass(Pairs{k % 2 ? keys : other_keys, k % 2 ? pos : other_pos}, k, p, hist, totals, to_keys, to_pos, part, s);
        }
        if (p.passes % 2 == 0) {
            keys = other_keys;
            pos = other_pos;
        }
        rc = launched("sort of tokens");
    };
    if (token_type == SCD_I32)
        sort(int32_t{});
    else
        sort(int64_t{});
    if (rc != SCD_OK || n == 0) return rc;
    SumArgs a{};
    a.keys = keys;
    a.pos = pos;
    a.n = p.n;
    a.share = p.share;
    a.rows = (uint32_t)rows;
    a.dim = (int32_t)dim;
    a.scale = scale;
    a.gstride = grad_stride;
    a.ostride = rows > 1 ? out_stride : dim;
    a.head = (float*)(w + (p.one ? 2 : 4) * p.pairs + p.hist);
    a.tail = (float*)((char*)a.head + p.pieces);
    with_vec(grad_type, out_type, dim, [&](auto tg, auto to, auto vc) {
        using TG = decltype(tg);
        using TO = decltype(to);
        constexpr int VEC = decltype(vc)::value;
        const RowMap m = row_map(dim, VEC);
        const dim3 grid((uint32_t)ceil_div(p.groups, kThreads >> m.log2_lanes), m.ranges);
        const auto go = [&](auto acc) {
            constexpr bool ACC = decltype(acc)::value;
            k_sums<VEC, ACC><<<grid, kThreads, 0, s>>>(a, (const TG*)grad, (TO*)out, m.log2_lanes);
            if (p.groups > 1) k_sums_join<VEC, ACC><<<grid, kThreads, 0, s>>>(a, (TO*)out, m.log2_lanes);
        };
        accumulate ? go(std::true_type{}) : go(std::false_type{});
    });
    return launched("scd_embed_grad");
}

// scd_embed.hip -- table lookup with scaling and its gradient by sorted tokens (gfx950).
//
// Lookup: out[t] = s E[tok[t]].  Gradient: dE[v] = s sum_{t: tok[t]=v} g[t].  Both only move data: the
// lookup reads the rows in use once and writes n rows; the gradient reads n rows and writes the whole table.
//
// The gradient sorts (token, position) pairs by token, stably, so that the rows of one token are consecutive and in
// ascending position; every run of equal tokens is then summed in registers and its row written once.  Runs are cut
// where a group of lanes or a workgroup has its share of the list; the pieces are added in 32 bits in an order that the
// sizes alone fix.  No floating-point atomics: results are bit-identical from call to call.  The zeros of the rows
// without a token are written by further workgroups of the sort's launches, which move little data themselves.
// Three ways to the sorted list, by its length: none at all (k_grad_few), tiles ordered by counting and merged
// (k_sort_tiles, k_sort_merge), a radix sort (k_sort_count, k_sort_scan, k_sort_move).
//
// Measured: 2.6 M ids looked up in 1.5 M x 16 (fp32) 50 us; gradients of 300 tokens into 4,999 x 777 8.8 us, of 16,384 into
// 75,000 x 1,024 (bf16) 42 us (sort with 154 MB of zeros 24, sums 12, join 5), of 1.28 M into 1.5 M x 16 (fp32)
// 110 us (sort with 96 MB of zeros 65, sums 39, join 8).
#include <algorithm>
#include <type_traits>

#include "scd_feat.h"

namespace scd {
namespace feat {
namespace {

// ---------------------------------------------------------------------------------------- lookup

// A large output goes past the caches (ONCE), so that the table's rows stay there.  2.6 M ids into 1.5 M x 16 (fp32, 164 MB
// out): 63 us through the caches, 53 past them; 16,384 x 4,096 (bf16, 134 MB): 42 and 34, and with the layer norm that
// reads them 88 and 86; but 4,096 x 4,096 (34 MB), which the norm then finds in the caches: 22.8 and 25.7 together.
// On both sides of the limit, alone and with a pass that reads the output at once: 80 MB of rows of 16 (fp32) 34 through
// and 24 past the caches, 50 and 53; 112 MB 47 and 33, 69 and 71.  The reader's loss falls from 8 % to 3 %, the lookup's gain
// stays.
constexpr int64_t kOnceBytes = int64_t(96) << 20;

template <int VEC, int U, bool ONCE, typename TI, typename TT, typename TO>
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
        if (g + u * groups < n) put_vec<ONCE>(out + (g + u * groups) * ostride + c, o);
    }
}

// ---------------------------------------------------------------------------------------- sort
// Keys are the tokens; one outside [0, rows) gets the key `rows` and so comes last.  The list is padded to a whole
// number of batches of k_sums with such keys, at position 0.

struct __align__(8) Pair {
    uint32_t key, pos;
};
static_assert(sizeof(Pair) == kPairBytes);

template <typename TI>
struct Tokens {
    const TI* tok;
    int64_t n;
    uint32_t rows;
    __device__ uint32_t key(int64_t i) const {
        const int64_t t = i < n ? (int64_t)tok[i] : -1;
        return t >= 0 && t < (int64_t)rows ? (uint32_t)t : rows;
    }
    __device__ Pair pair(int64_t i) const { return Pair{key(i), i < n ? (uint32_t)i : 0}; }
};
struct Pairs {
    const Pair* p;
    __device__ uint32_t key(int64_t i) const { return p[i].key; }
    __device__ Pair pair(int64_t i) const { return p[i]; }
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
        const Piece piece = fill_piece(f.rows * f.row_bytes, block, blocks);
        fill_bytes(f.p + piece.from, piece.bytes, threadIdx.x, blockDim.x);
        return;
    }
    const int64_t waves = (int64_t)blocks * (blockDim.x / 64);
    for (int64_t r = (int64_t)block * (blockDim.x / 64) + threadIdx.x / 64; r < f.rows; r += waves)
        fill_bytes(f.p + r * f.stride, f.row_bytes, threadIdx.x % 64, 64);
}

// The lanes of the wave that hold the same digit as this one, among the active ones.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits) {
    const uint64_t all = __ballot(1);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
    for (int b = 0; b < bits; ++b) {
        const uint32_t mine = (uint32_t)((int32_t)(digit << (31 - b)) >> 31);  // all ones where the bit is set
        const uint64_t set = __ballot(mine != 0);
        lo &= ~((uint32_t)set ^ mine);
        hi &= ~((uint32_t)(set >> 32) ^ mine);
    }
    return (uint64_t)hi << 32 | lo;
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
                                           uint16_t* counts, uint32_t (&rank)[J]) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (!on[j]) continue;
        const uint64_t m = same_digit(digit[j], bits);
        const uint32_t below = lanes_below(m);
        const uint32_t base = counts[digit[j]];
        rank[j] = base + below;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // LDS serves a wave's accesses in order
        if (below == 0) counts[digit[j]] = (uint16_t)(base + (uint32_t)__popcll(m));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Short lists, in two launches without passes.  k_sort_tiles orders tiles of 256 entries, an entry's place being the
// number of entries of its tile before it, counted: each wave compares 64 entries, one to a lane, with 64 others.
// k_sort_merge then places every entry in the whole list: its place is the sum over the tiles of the entries before it,
// which a binary search in each finds (those of equal key count in the tiles before its own).  A workgroup of
// k_sort_merge holds all keys in LDS and places kMergeEntries entries, two to a lane; each of its waves searches a
// sixteenth of the tiles, four at a time.
constexpr int kMergeThreads = 1024;
constexpr int kMergeWaves = kMergeThreads / 64;
constexpr int kMergeEntries = 128;

template <typename TI>
__global__ void __launch_bounds__(4 * kSmallTile) k_sort_tiles(Tokens<TI> src, uint32_t n, Pair* __restrict__ pairs,
                                                               uint32_t* __restrict__ sorted_keys, uint32_t tiles, Fill fill) {
    if (blockIdx.x >= tiles) {
        fill_zero(fill, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    __shared__ __align__(16) uint32_t keys[kSmallTile];
    __shared__ uint32_t counts[4][kSmallTile];
    const uint32_t at = threadIdx.x % kSmallTile, part = threadIdx.x / kSmallTile, own = at / 64;
    const uint32_t i = blockIdx.x * kSmallTile + at;
    const Pair p = src.pair(i);
    if (part == 0) keys[at] = i < n ? p.key : 0xFFFFFFFFu;  // above every key
    __syncthreads();
    uint32_t before = 0;
    if (part == own) {
#pragma unroll 8
        for (uint32_t k = 0; k < 64; ++k) {
            const uint32_t q = keys[part * 64 + k];
            before += q < p.key || (q == p.key && k < at % 64);
        }
    } else {
        const uint32_t bound = p.key + (part < own);
#pragma unroll
        for (uint32_t k = 0; k < 16; ++k) {
            const uint4 q = reinterpret_cast<const uint4*>(keys + part * 64)[k];
            before += (q.x < bound) + (q.y < bound) + (q.z < bound) + (q.w < bound);
        }
    }
    counts[part][at] = before;
    __syncthreads();
    if (part == 0) {
        const uint32_t to = blockIdx.x * kSmallTile + counts[0][at] + counts[1][at] + counts[2][at] + counts[3][at];
        if (i < n) pairs[to] = p;
        sorted_keys[i < n ? to : i] = keys[at];  // whole tiles
    }
}

__global__ void __launch_bounds__(kMergeThreads) k_sort_merge(const Pair* __restrict__ in, const uint32_t* __restrict__ sorted_keys,
                                                              uint32_t n, Pair* __restrict__ out, uint32_t own_blocks, Fill fill) {
    if (blockIdx.x >= own_blocks) {
        fill_zero(fill, blockIdx.x - own_blocks, gridDim.x - own_blocks);
        return;
    }
    constexpr int U = 4, E = kMergeEntries / 64;
    extern __shared__ __align__(16) uint32_t keys[];  // whole tiles, then a count per wave and entry
    const uint32_t tiles = (n + kSmallTile - 1) / kSmallTile, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t* const counts = keys + tiles * kSmallTile;
    // A workgroup's entries lie in one tile.
    const uint32_t first = blockIdx.x * kMergeEntries + lane, own = blockIdx.x * kMergeEntries / kSmallTile;
    Pair p[E];
    uint32_t before[E] = {};
#pragma unroll
    for (int k = 0; k < E; ++k) p[k] = in[min(first + k * 64, n - 1)];
    for (uint32_t k = threadIdx.x; k < tiles * kSmallTile / 4; k += kMergeThreads)
        reinterpret_cast<uint4*>(keys)[k] = reinterpret_cast<const uint4*>(sorted_keys)[k];
    __syncthreads();
    for (uint32_t t = wave; t < tiles; t += U * kMergeWaves) {
        uint32_t at[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < E; ++k) at[u][k] = 0;
#pragma unroll
        for (uint32_t step = kSmallTile / 2; step; step /= 2)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t q = min(t + u * kMergeWaves, tiles - 1);
#pragma unroll
                for (int k = 0; k < E; ++k) at[u][k] += keys[q * kSmallTile + at[u][k] + step - 1] < p[k].key + (q < own) ? step : 0;
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t q = t + u * kMergeWaves;
            if (q >= tiles || q == own) continue;
#pragma unroll
            for (int k = 0; k < E; ++k) before[k] += at[u][k] + (keys[q * kSmallTile + at[u][k]] < p[k].key + (q < own));
        }
    }
#pragma unroll
    for (int k = 0; k < E; ++k) counts[(wave * E + k) * 64 + lane] = before[k];
    __syncthreads();
    if (wave < E && first + wave * 64 < n) {
        uint32_t to = (first + wave * 64) % kSmallTile;
#pragma unroll
        for (int w = 0; w < kMergeWaves; ++w) to += counts[(w * E + wave) * 64 + lane];
        out[to] = wave ? p[E - 1] : p[0];
    }
}
static_assert(kMergeEntries == 128 && kSmallTile % kMergeEntries == 0, "two entries a lane, of one tile");

// Long lists: a radix sort from the lowest digit up, a workgroup for each tile of kTileThreads x J consecutive entries.  A pass
// counts the tiles' digits (k_sort_count), sums the counts along the tiles (k_sort_scan), and moves the entries
// (k_sort_move), which orders its tile in LDS first, so that it writes runs of consecutive entries.  Every launch
// fills a part of the zeros with further workgroups.  The move is bound by its tiles' counters (one for each wave and
// digit): 1.28 M entries in digits of 11 bits take 17 to 20 us, in which their stores take 3.
constexpr int kTileWaves = kTileThreads / 64;
constexpr int kPer = (1 << kMaxBits) / kTileThreads;  // digits a thread at most: k_sort_move gives it consecutive ones

template <int J, typename SRC>
__global__ void __launch_bounds__(kTileThreads) k_sort_count(SRC src, int64_t n, int shift, int bits, uint32_t tiles,
                                                             uint32_t* __restrict__ hist, Fill fill) {
    if (blockIdx.x >= tiles) {
        fill_zero(fill, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    __shared__ uint32_t count[1 << kMaxBits];
    const uint32_t bins = 1u << bits;
    for (uint32_t d = threadIdx.x; d < bins; d += kTileThreads) count[d] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * (kTileThreads * J);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int64_t i = base + j * kTileThreads + threadIdx.x;
        if (i < n) atomicAdd(&count[(src.key(i) >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < bins; d += kTileThreads) hist[((int64_t)blockIdx.x << bits) + d] = count[d];
}

// hist[tile][digit] becomes the digit's count in the tiles before, totals[digit] its count in all: kScanDigits digits a
// workgroup, the tiles in kScanSlices runs.
constexpr int kScanDigits = 16;
constexpr int kScanSlices = 64;

__global__ void __launch_bounds__(kScanDigits * kScanSlices) k_sort_scan(uint32_t* __restrict__ hist, uint32_t tiles, int bits,
                                                                uint32_t* __restrict__ totals, uint32_t own_blocks, Fill fill) {
    if (blockIdx.x >= own_blocks) {
        fill_zero(fill, blockIdx.x - own_blocks, gridDim.x - own_blocks);
        return;
    }
    constexpr int U = 8;
    __shared__ uint32_t sums[kScanSlices][kScanDigits];
    const uint32_t lane = threadIdx.x % kScanDigits, slice = threadIdx.x / kScanDigits, d = blockIdx.x * kScanDigits + lane;
    const bool on = d < 1u << bits;
    const uint32_t t0 = (uint32_t)((uint64_t)tiles * slice / kScanSlices), t1 = (uint32_t)((uint64_t)tiles * (slice + 1) / kScanSlices);
    uint32_t x[U], sum = 0;
    const auto fetch = [&](uint32_t t) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = on && t + u < t1 ? hist[((int64_t)(t + u) << bits) + d] : 0;
    };
    for (uint32_t t = t0; t < t1; t += U) {
        fetch(t);
#pragma unroll
        for (int u = 0; u < U; ++u) sum += x[u];
    }
    sums[slice][lane] = sum;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll 16
    for (uint32_t k = 0; k < kScanSlices; ++k) {
        const uint32_t y = sums[k][lane];
        before += k < slice ? y : 0;
        total += y;
    }
    for (uint32_t t = t0; t < t1; t += U) {
        if (t1 - t0 > U) fetch(t);  // a run of up to U tiles is still there
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (on && t + u < t1) {
                hist[((int64_t)(t + u) << bits) + d] = before;
                before += x[u];
            }
    }
    if (on && slice == 0) totals[d] = total;
}

template <int J, typename SRC>
__global__ void __launch_bounds__(kTileThreads) k_sort_move(SRC src, int64_t n, int shift, int bits, uint32_t tiles,
                                                            const uint32_t* __restrict__ hist,
                                                            const uint32_t* __restrict__ totals, Pair* __restrict__ out, Fill fill) {
    if (blockIdx.x >= tiles) {
        fill_zero(fill, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    constexpr int kTile = kTileThreads * J;
    __shared__ Pair tile[kTile];
    extern __shared__ __align__(16) uint32_t shift_of[];              // [digit]: from a place in the ordered tile to that in `out`
    uint16_t* const counts = reinterpret_cast<uint16_t*>(shift_of + (1 << bits));  // [wave][digit]
    __shared__ uint32_t sums[kTileWaves];
    const uint32_t bins = 1u << bits, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t per = max(1u, bins / kTileThreads), d0 = threadIdx.x * per;
    for (uint32_t i = threadIdx.x; i < kTileWaves * bins / 2; i += kTileThreads) reinterpret_cast<uint32_t*>(counts)[i] = 0;
    const int64_t base = (int64_t)blockIdx.x * kTile, at = base + wave * 64 * J + lane;
    Pair p[J];
    uint32_t digit[J], rank[J], all = 0, total;
    bool on[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int64_t i = at + j * 64;
        on[j] = i < n;
        p[j] = src.pair(on[j] ? i : 0);
        digit[j] = (p[j].key >> shift) & (bins - 1);
    }
    // Where the digits of this thread begin in `out`: the smaller digits' totals and the tiles before.
    uint32_t t[kPer], earlier[kPer];
#pragma unroll
    for (uint32_t k = 0; k < kPer; ++k) {
        const bool mine = k < per && d0 + k < bins;
        t[k] = mine ? totals[d0 + k] : 0;
        earlier[k] = mine ? hist[((int64_t)blockIdx.x << bits) + d0 + k] : 0;
        all += t[k];
    }
    uint32_t start = block_exclusive(all, sums, total);
    wave_ranks<J>(digit, on, bits, counts + wave * bins, rank);
    __syncthreads();
    uint32_t here[kPer], sum = 0;
#pragma unroll
    for (uint32_t k = 0; k < kPer; ++k) {
        here[k] = 0;
        if (k < per && d0 + k < bins)
#pragma unroll
            for (int w = 0; w < kTileWaves; ++w) here[k] += counts[w * bins + d0 + k];
        sum += here[k];
    }
    uint32_t first = block_exclusive(sum, sums, total);
#pragma unroll
    for (uint32_t k = 0; k < kPer; ++k)
        if (k < per && d0 + k < bins) {
            shift_of[d0 + k] = start + earlier[k] - first;
            start += t[k];
            uint32_t to = first;
#pragma unroll
            for (int w = 0; w < kTileWaves; ++w) {
                const uint32_t c = counts[w * bins + d0 + k];
                counts[w * bins + d0 + k] = (uint16_t)to;
                to += c;
            }
            first = to;
        }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (on[j]) tile[counts[wave * bins + digit[j]] + rank[j]] = p[j];
    __syncthreads();
    const uint32_t entries = (uint32_t)min((int64_t)kTile, n - base);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t i = j * kTileThreads + threadIdx.x;
        if (i < entries) {
            const Pair q = tile[i];
            out[i + shift_of[(q.key >> shift) & (bins - 1)]] = q;
        }
    }
}

// ---------------------------------------------------------------------------------------- sums
// A group of lanes sums `share` consecutive entries of the sorted list, run by run; a run that lies inside is final.  The
// pieces of a run that goes over several groups of a workgroup are added in LDS by the group where it ends.  Of a run
// that goes over several workgroups, the one where it ends keeps its piece in head[workgroup], those before theirs in
// tail[workgroup], and k_sums_join adds them in order.  All pieces are 32 bits and unscaled.  Bound by the gathers:
// 16,384 rows of 2 KB in 12 us (2.8 TB/s, 33.5 MB), 1.28 M rows of 64 bytes in 39 us (2.1 TB/s); the join is a chain
// of four dependent reads, 5 us.

struct SumArgs {
    const Pair* pairs;
    int64_t n;
    uint32_t share;  // entries of a group
    uint32_t block;  // entries of a workgroup of k_sums
    // Gradients are read past the caches, but not rows that share a 64-byte line with others.  Whole calls, past and through
    // the caches: 16,384 tokens into 75,000 x 1,024 (bf16) 43 and 49 us, 1.28 M into 1.5 M x 16 (fp32) 113 and 122;
    // 1.28 M into 1.5 M x 16 in bf16 120 and 115.
    bool once;
    bool flat;  // k_grad_few: fills pieces of memory, not rows
    uint32_t rows;
    int32_t dim;
    float scale;
    int64_t gstride, ostride;
    float* head;  // [workgroups of k_sums][dim]
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

template <int VEC, bool ACC, int THREADS, typename TG, typename TO>
__global__ void __launch_bounds__(THREADS) k_sums(SumArgs a, const TG* __restrict__ grad, TO* __restrict__ out, uint32_t log2_lanes) {
    constexpr int U = kBatch;  // divides the share and the list
    __shared__ float tails[THREADS * VEC];
    __shared__ uint32_t begins[THREADS / 32];  // a bit by group: what it hands on begins there (else it is a run's middle part)
    for (uint32_t k = threadIdx.x; k < THREADS / 32; k += THREADS) begins[k] = 0;
    __syncthreads();
    const uint32_t j = threadIdx.x >> log2_lanes, l = threadIdx.x & ((1u << log2_lanes) - 1);
    const int32_t col = (int32_t)((blockIdx.y << log2_lanes) + l);
    const bool in = col * VEC < a.dim;
    int32_t again;
    const int32_t c = vec_column<VEC>(in ? col : 0, a.dim, again);
    const int64_t e0 = (int64_t)blockIdx.x * a.block + j * a.share, e1 = min(a.n, e0 + a.share);
    uint32_t cur = 0, opening = 0;
    bool cut = false, has_head = false, more = false;
    float acc[VEC] = {}, head[VEC] = {};
    if (e0 < a.n) {
        cur = opening = a.pairs[e0].key;
        cut = e0 > 0 && a.pairs[e0 - 1].key == cur;
        const uint32_t after = a.pairs[min(e1, a.n - 1)].key;
        for (int64_t e = e0; e < e1; e += U) {
            const Raw<U, Pair> p = load_raw<U>(a.pairs + e);
            Raw<VEC, TG> v[U];
            if (a.once) {
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = load_raw_once<VEC>(grad + (int64_t)p.t[u].pos * a.gstride + c);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = load_raw<VEC>(grad + (int64_t)p.t[u].pos * a.gstride + c);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p.t[u].key != cur) {
                    if (cut) {
                        has_head = true;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) head[i] = acc[i];
                    } else if (in) {
                        write_row<VEC, ACC>(a, out, cur, c, again, acc);
                    }
                    cut = false;
                    cur = p.t[u].key;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
                }
                float x[VEC];
                widen(v[u], x);
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] += x[i];
            }
        }
        if (cur < a.rows) {
            more = e1 < a.n && after == cur;
            if (!more && cut) {
                has_head = true;
#pragma unroll
                for (int i = 0; i < VEC; ++i) head[i] = acc[i];
            } else if (!more && in) {
                write_row<VEC, ACC>(a, out, cur, c, again, acc);
            }
        }
    }
    if (l == 0 && !(more && cut)) atomicOr(&begins[j / 32], 1u << j % 32);
#pragma unroll
    for (int i = 0; i < VEC; ++i) tails[threadIdx.x * VEC + i] = acc[i];
    __syncthreads();
    // Adds the pieces of the run that group j - 1 hands on, from the group where it begins; true where that lies before the
    // workgroup.
    const auto add_before = [&](float (&s)[VEC]) {
        int32_t word = (int32_t)j / 32;
        uint32_t bits = begins[word] & ((1u << j % 32) - 1);
        while (!bits && word > 0) bits = begins[--word];
        const bool open = !bits;
        for (uint32_t k = open ? 0 : word * 32 + 31 - __builtin_clz(bits); k < j; k += U) {
            float x[U][VEC];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < VEC; ++i) x[u][i] = tails[((min(k + u, j - 1) << log2_lanes) + l) * VEC + i];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[i] += k + u < j ? x[u][i] : 0.0f;
        }
        return open;
    };
    if (!in) return;
    if (has_head) {
        float s[VEC] = {};
        const bool open = add_before(s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] += head[i];
        if (open)
            store_vec(a.head + (int64_t)blockIdx.x * a.dim + c, s);
        else
            write_row<VEC, ACC>(a, out, opening, c, again, s);
    }
    if (more && j == (THREADS >> log2_lanes) - 1) {  // the run goes on in the next workgroup
        float s[VEC] = {};
        if (cut) add_before(s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] += acc[i];
        store_vec(a.tail + (int64_t)blockIdx.x * a.dim + c, s);
    }
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

// The workgroup of k_sums in which the run that covers the start of its workgroup g (and the entry before it) begins.  The
// starts of the workgroups 1, 2, 4, ... before are looked at, several together, then the range between two of them in eighths.
__device__ __forceinline__ int64_t run_begins(const SumArgs& a, int64_t g, uint32_t row) {
    constexpr int P = 8;
    const auto covers = [&](int64_t k, uint32_t key) { return k > 0 && key == row; };
    const auto before = [&](int64_t k) { return a.pairs[max(k, (int64_t)1) * a.block - 1].key; };
    int64_t in = g, out = 0;  // the run covers the start of `in`; once out < in, not that of `out`
    bool more = true;
    const auto probe = [&](auto probes, int64_t step) {  // looks at g - step, g - 2 step, g - 4 step, ... together
        constexpr int N = decltype(probes)::value;
        uint32_t key[N];
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = before(g - (step << i));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t k = g - (step << i);
            if (more && covers(k, key[i])) {
                in = k;
            } else if (more) {
                out = max(k, (int64_t)0);
                more = false;
            }
        }
    };
    probe(Int<2>{}, 1);  // most runs are short
    int64_t step = 4;
    while (more) {
        probe(Int<P>{}, step);
        step <<= P;
    }
    while (in - out > 1) {  // the run's first entry lies in a workgroup from `out` to in - 1
        const int64_t lo = out, size = in - out;
        uint32_t key[P - 1];
#pragma unroll
        for (int i = 1; i < P; ++i) key[i - 1] = before(lo + max((int64_t)1, size * i / P));
#pragma unroll
        for (int i = P - 1; i >= 1; --i) {
            const int64_t k = lo + max((int64_t)1, size * i / P);
            if (covers(k, key[i - 1])) in = min(in, k);
        }
#pragma unroll
        for (int i = 1; i < P; ++i) {
            const int64_t k = lo + max((int64_t)1, size * i / P);
            if (!covers(k, key[i - 1])) out = max(out, k);
        }
    }
    return out;
}

// A group of lanes for each workgroup of k_sums: where a run ends there that began before, it joins the run's pieces.  Of
// many pieces, each of the m groups of its wave (or, where a wave has one group or the run is very long, of its workgroup)
// adds every m-th, and the m sums are added in a fixed order.
template <int VEC, bool ACC, int THREADS, typename TO>
__global__ void __launch_bounds__(THREADS) k_sums_join(SumArgs a, TO* __restrict__ out, uint32_t log2_lanes) {
    __shared__ float part[THREADS * VEC];
    __shared__ int64_t ends[THREADS], begins[THREADS];
    const uint32_t m = THREADS >> log2_lanes, j = threadIdx.x >> log2_lanes, l = threadIdx.x & ((1u << log2_lanes) - 1);
    const int64_t g = (int64_t)blockIdx.x * m + j;
    const int32_t col = (int32_t)((blockIdx.y << log2_lanes) + l);
    const bool in = col * VEC < a.dim;
    int32_t again;
    const int32_t c = vec_column<VEC>(in ? col : 0, a.dim, again);
    const int64_t e0 = g * a.block, e1 = min(a.n, e0 + a.block);
    int64_t begin = -1;
    uint32_t row = 0;
    if (e0 > 0 && e0 < a.n) {
        const uint32_t before = a.pairs[e0 - 1].key, after = a.pairs[min(e1, a.n - 1)].key;
        row = a.pairs[e0].key;
        if (row < a.rows && before == row && (e1 == a.n || after != row)) begin = run_begins(a, g, row);
    }
    const int64_t pieces = begin >= 0 ? g - begin : 0;
    const uint32_t beside = log2_lanes < 6 ? 64 >> log2_lanes : 1;  // groups in a wave
    const bool is_long = pieces > (beside > 1 ? 32 * beside : 16), is_wave = !is_long && beside > 1 && pieces > 16;
    if (l == 0) {
        ends[j] = is_long ? g : -1;
        begins[j] = begin;
    }
    for (uint64_t todo = __ballot(is_wave && l == 0); todo; todo &= todo - 1) {
        const int at = __builtin_ctzll(todo);
        const int64_t last = __shfl((int)g, at), from = __shfl((int)begin, at);
        float s[VEC] = {};
        if (in) add_tails<VEC>(a, from + j % beside, last, beside, c, s);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            for (int o = 32; o >= 1 << log2_lanes; o /= 2) s[i] += __shfl_xor(s[i], o);
        if (g == last && in) {
            const Raw<VEC, float> h = load_raw<VEC>(a.head + g * a.dim + c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[i] += h.t[i];
            write_row<VEC, ACC>(a, out, row, c, again, s);
        }
    }
    if (begin >= 0 && !is_long && !is_wave && in) {
        float s[VEC] = {};
        const Raw<VEC, float> h = load_raw<VEC>(a.head + g * a.dim + c);
        add_tails<VEC>(a, begin, g, 1, c, s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] += h.t[i];
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
            write_row<VEC, ACC>(a, out, a.pairs[end * a.block].key, c, again, s);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------- few tokens
// With at most kFewMax tokens one launch does it all: a workgroup owns some consecutive rows (and, of wide ones, a column
// range), picks the tokens that lie in them, orders them by counting, fills the other rows with zeros and sums the runs,
// long ones with several groups.  Every workgroup reads all tokens, so this is for lists that cost less than
// the launches of a sort.  1,024 tokens, one to each thread, are where it ends: they still take less than by the sort
// (75,000 x 1,024 in bf16 32 and 39 us, 1.5 M x 16 in fp32 19 and 27, 1,000 x 64 in fp32 10 and 16).
constexpr int kFewThreads = 1024;
static_assert(kFewMax <= kFewThreads, "a thread holds a token");
constexpr int kFewRows = 16384;  // of a workgroup at most: a bit each in LDS
constexpr int64_t kFlatBytes = int64_t(64) << 20;

template <int VEC, bool ACC, typename TI, typename TG, typename TO>
__global__ void __launch_bounds__(kFewThreads) k_grad_few(Tokens<TI> src, SumArgs a, const TG* __restrict__ grad, TO* __restrict__ out,
                                                          uint32_t own_rows, uint32_t log2_lanes) {
    constexpr int U = 8;
    __shared__ uint32_t given[kFewRows / 32];    // the rows that have tokens
    __shared__ __align__(16) uint32_t keys[kFewMax];
    __shared__ uint32_t places[kFewMax];
    __shared__ Pair sorted[kFewMax];
    __shared__ uint32_t starts[kFewMax + 1], sums[kFewThreads / 64];
    __shared__ float part[kFewThreads * VEC];
    const uint32_t r0 = blockIdx.x * own_rows, here = min(own_rows, a.rows - r0), i = threadIdx.x;
    const uint32_t m = kFewThreads >> log2_lanes, j = i >> log2_lanes, l = i & ((1u << log2_lanes) - 1);
    const int32_t col = (int32_t)((blockIdx.y << log2_lanes) + l);
    const bool in = col * VEC < a.dim;
    int32_t again;
    const int32_t c = vec_column<VEC>(in ? col : 0, a.dim, again);
    for (uint32_t k = i; k < (here + 31) / 32; k += kFewThreads) given[k] = 0;
    const uint32_t key = i < src.n ? src.key(i) - r0 : here;
    const bool mine = key < here;  // also false for keys below r0, which wrap
    uint32_t count, runs;
    keys[i] = 0xFFFFFFFFu;  // above every key; block_exclusive waits for all
    uint32_t at = block_exclusive(mine, sums, count);
    if (mine) {
        keys[at] = key;
        places[at] = i;
        atomicOr(&given[key / 32], 1u << key % 32);
    }
    __syncthreads();
    const auto fill_others = [&] {
        if (ACC) return;
        if (a.flat) {
            // The rows between two that have tokens are one piece of memory: the workgroup fills one after another, or,
            // where they are many, each of its waves one.  The column ranges' workgroups share it.
            const int64_t row_bytes = (int64_t)a.dim * (int64_t)sizeof(TO);
            const bool all = runs < kFewThreads / 64;
            for (uint32_t q = all ? 0 : i / 64; q <= runs; q += all ? 1 : kFewThreads / 64) {
                const uint32_t lo = q ? sorted[starts[q - 1]].key + 1 : 0, hi = q < runs ? sorted[starts[q]].key : here;
                const int64_t total = (int64_t)(hi - lo) * row_bytes, from = total * blockIdx.y / gridDim.y / 64 * 64;
                const int64_t to = blockIdx.y + 1 < gridDim.y ? total * (blockIdx.y + 1) / gridDim.y / 64 * 64 : total;
                fill_bytes((char*)out + (int64_t)(r0 + lo) * row_bytes + from, to - from, all ? i : i % 64, all ? kFewThreads : 64);
            }
            return;
        }
        if (!in) return;
        const float zero[VEC] = {};
        for (uint32_t r = j; r < here; r += m)
            if (!(given[r / 32] >> r % 32 & 1)) store_vec(out + (int64_t)(r0 + r) * a.ostride + c, zero);
    };
    if (count == 0) {
        runs = 0;
        fill_others();
        return;
    }
    if (i < count) {  // its place: how many of the keys before it in the list are at most its key, and of those after it less
        const uint32_t own = keys[i], wave = i / 64;
        uint32_t to = 0;
        for (uint32_t b = 0; b * 64 < count; ++b) {
            if (b != wave) {
                const uint4* const q = reinterpret_cast<const uint4*>(keys + b * 64);
                const uint32_t bound = own + (b < wave);
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) to += (q[k].x < bound) + (q[k].y < bound) + (q[k].z < bound) + (q[k].w < bound);
            } else {
                const uint32_t last = min(64u, count - b * 64);
                for (uint32_t k = 0; k < last; ++k) to += keys[b * 64 + k] < own + (k < i % 64);
            }
        }
        sorted[to] = Pair{own, places[i]};
    }
    __syncthreads();
    const bool start = i < count && (i == 0 || sorted[i].key != sorted[i - 1].key);
    at = block_exclusive(start, sums, runs);
    if (start) starts[at] = i;
    if (i == 0) starts[runs] = count;
    __syncthreads();
    fill_others();  // after the last barrier of the ordering, which would wait for the stores
    const auto add = [&](uint32_t from, uint32_t end, uint32_t step, float (&s)[VEC]) {
        for (uint32_t e = from; e < end; e += U * step) {
            Raw<VEC, TG> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_raw<VEC>(grad + (int64_t)sorted[min(e + u * step, end - 1)].pos * a.gstride + c);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[VEC];
                widen(v[u], x);
#pragma unroll
                for (int k = 0; k < VEC; ++k) s[k] += e + u * step < end ? x[k] : 0.0f;
            }
        }
    };
    constexpr uint32_t kLong = 2 * U;  // entries that a group sums alone
    for (uint32_t q = j; q < runs && in; q += m) {
        const uint32_t from = starts[q], end = starts[q + 1];
        if (end - from > kLong) continue;
        float s[VEC] = {};
        add(from, end, 1, s);
        write_row<VEC, ACC>(a, out, r0 + sorted[from].key, c, again, s);
    }
    if (log2_lanes < 6) {  // a wave for each longer run
        const uint32_t beside = 64 >> log2_lanes;
        for (uint32_t q = i / 64; q < runs; q += kFewThreads / 64) {
            const uint32_t from = starts[q], end = starts[q + 1];
            if (end - from <= kLong) continue;
            float s[VEC] = {};
            if (in && from + j % beside < end) add(from + j % beside, end, beside, s);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                for (int o = 32; o >= 1 << log2_lanes; o /= 2) s[k] += __shfl_xor(s[k], o);
            if (j % beside == 0 && in) write_row<VEC, ACC>(a, out, r0 + sorted[from].key, c, again, s);
        }
        return;
    }
    // m is from 4 to 16 here, less than such a run has entries.
    for (uint32_t q = 0; q < runs; ++q) {
        const uint32_t from = starts[q], end = starts[q + 1];
        if (end - from <= kLong) continue;
        float s[VEC] = {};
        if (in) add(from + j, end, m, s);
#pragma unroll
        for (int k = 0; k < VEC; ++k) part[i * VEC + k] = s[k];
        __syncthreads();
        if (j == 0 && in) {
            for (uint32_t k = 1; k < m; ++k)
#pragma unroll
                for (int v = 0; v < VEC; ++v) s[v] += part[((k << log2_lanes) + l) * VEC + v];
            write_row<VEC, ACC>(a, out, r0 + sorted[from].key, c, again, s);
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

// Workgroups of `threads` threads that fill a part of the zeros beside other work: 64 bytes a thread, but at most 2 M
// threads in all.
uint32_t fill_blocks(const Fill& f, int threads) {
    if (!f.p) return 0;
    return (uint32_t)std::min<int64_t>(ceil_div(f.rows * f.row_bytes, threads * 64), 2048 * (1024 / threads));
}

// The first `part` of `parts` equal parts, the second, ...
Fill fill_part(const Fill& f, int64_t part, int64_t parts) {
    const int64_t a = f.rows * part / parts, b = f.rows * (part + 1) / parts;
    return f.p && b > a ? Fill{f.p + a * f.stride, b - a, f.row_bytes, f.stride} : Fill{};
}

// Leaves the sorted list in `pairs`; `other` is scratch.
template <typename TI>
int sort_short(Tokens<TI> src, const Plan& p, Pair* pairs, Pair* other, uint32_t* keys, const Fill& fill, hipStream_t s) {
    const uint32_t tiles = (uint32_t)ceil_div(p.n, kSmallTile), blocks = (uint32_t)ceil_div(p.n, kMergeEntries);
    Fill part = fill_part(fill, 0, 2);
    k_sort_tiles<<<tiles + fill_blocks(part, 4 * kSmallTile), 4 * kSmallTile, 0, s>>>(src, (uint32_t)p.n, other, keys, tiles, part);
    const size_t lds = (size_t)(tiles * kSmallTile + kMergeWaves * kMergeEntries) * 4;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_sort_merge), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return fail(SCD_ERR_HIP, "hipFuncSetAttribute: %s", hipGetErrorString(e));
    }
    part = fill_part(fill, 1, 2);
    k_sort_merge<<<blocks + fill_blocks(part, kMergeThreads), kMergeThreads, lds, s>>>(other, keys, (uint32_t)p.n, pairs, blocks, part);
    return launched("sort of tokens");
}

template <int J, typename SRC>
void launch_pass(SRC src, int pass, const Plan& p, uint32_t* hist, uint32_t* totals, Pair* out, const Fill* fills, hipStream_t s) {
    const uint32_t tiles = (uint32_t)p.tiles, scans = (uint32_t)ceil_div(1 << p.bits, kScanDigits);
    const int shift = pass * p.bits;
    k_sort_count<J><<<tiles + fill_blocks(fills[0], kTileThreads), kTileThreads, 0, s>>>(src, p.n, shift, p.bits, tiles, hist, fills[0]);
    k_sort_scan<<<scans + fill_blocks(fills[1], kScanDigits * kScanSlices), kScanDigits * kScanSlices, 0, s>>>(hist, tiles, p.bits, totals, scans, fills[1]);
    k_sort_move<J><<<tiles + fill_blocks(fills[2], kTileThreads), kTileThreads, (4 + 2 * kTileWaves) << p.bits, s>>>(src, p.n, shift, p.bits, tiles, hist, totals, out, fills[2]);
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
    const int U = embed_unroll(n, m);
    const int64_t most = embed_tokens(m, U);
    with_vec(table_type, out_type, dim, [&](auto tt, auto to, auto vc) {
        using TT = decltype(tt);
        using TO = decltype(to);
        constexpr int VEC = decltype(vc)::value;
        const auto go = [&](auto ti, auto uc, auto once) {
            using TI = decltype(ti);
            constexpr int U = decltype(uc)::value;
            for (int64_t from = 0; from < n; from += most) {
                const int64_t here = std::min(most, n - from);
                const dim3 grid((uint32_t)ceil_div(here, (kThreads >> m.log2_lanes) * U), m.ranges);
                k_embed<VEC, U, decltype(once)::value><<<grid, kThreads, 0, (hipStream_t)stream>>>(
                    (const TI*)tokens + from, here, (const TT*)table, table_stride, rows, (int32_t)dim, scale, (TO*)out + from * out_stride, out_stride,
                    m.log2_lanes);
            }
        };
        const auto with_ids = [&](auto ti) {
            if (U == 1)
                go(ti, Int<1>{}, std::false_type{});
            else if (n * dim * type_bytes(out_type) < kOnceBytes)
                go(ti, Int<4>{}, std::false_type{});
            else
                go(ti, Int<4>{}, std::true_type{});
        };
        token_type == SCD_I32 ? with_ids(int32_t{}) : with_ids(int64_t{});
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
    const Plan p = plan_for(n, rows, dim);
    if (p.bytes && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < p.bytes))
        return fail(SCD_ERR_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)p.bytes);
    SumArgs a{};
    a.rows = (uint32_t)rows;
    a.dim = (int32_t)dim;
    a.scale = scale;
    a.gstride = grad_stride;
    a.ostride = rows > 1 ? out_stride : dim;
    if (p.few) {
        with_vec(grad_type, out_type, dim, [&](auto tg, auto to, auto vc) {
            using TG = decltype(tg);
            using TO = decltype(to);
            constexpr int VEC = decltype(vc)::value;
            const RowMap m = row_map(dim, VEC);
            // A workgroup's rows: as many as let 512 workgroups, two to a CU, share the table, but 16 KB at least.
            const int64_t least = ceil_div(16384, ((int64_t)VEC << m.log2_lanes) * (int64_t)sizeof(TO));
            const int64_t own = std::min<int64_t>(kFewRows, std::max(least, ceil_div(rows * m.ranges, 512)));
            const dim3 grid((uint32_t)ceil_div(rows, own), m.ranges);
            // A large table without gaps between its rows: 3 tokens into 75,829 x 1,055 (fp32) 95 us by rows, 75 by pieces;
            // 300 into 4,999 x 777 8.7 and 10.6.  Pieces gain where rows come in ranges that end inside a line, and lose time
            // to many tokens: 3, 300 and 1,000 tokens into 1,055 columns 11.0, 13.7 and 16.0 us by rows and 10.2, 15.4 and
            // 22.0 by pieces at 32 MB, 14.5, 17.2, 19.9 and 12.5, 17.1, 23.8 at 64 MB, 20.9, 24.0, 27.3 and 18.1, 20.8, 27.0
            // at 96 MB; 777 columns at 64 MB 12.6, 14.5, 16.6 and 13.1, 15.9, 18.7, at 320 MB 85, 86, 88 and 76, 80, 85.
            a.flat = a.ostride == dim && rows * dim * (int64_t)sizeof(TO) >= kFlatBytes;
            const auto go = [&](auto ti, auto acc) {
                using TI = decltype(ti);
                k_grad_few<VEC, decltype(acc)::value><<<grid, kFewThreads, 0, s>>>(Tokens<TI>{(const TI*)tokens, n, (uint32_t)rows}, a, (const TG*)grad, (TO*)out, (uint32_t)own, m.log2_lanes);
            };
            if (token_type == SCD_I32)
                accumulate ? go(int32_t{}, std::true_type{}) : go(int32_t{}, std::false_type{});
            else
                accumulate ? go(int64_t{}, std::true_type{}) : go(int64_t{}, std::false_type{});
        });
        return launched("scd_embed_grad");
    }
    Fill fill{};
    if (!accumulate) fill = Fill{(char*)out, rows, dim * e, rows > 1 ? out_stride * e : dim * e};
    char* w = (char*)workspace;
    Pair* pairs = (Pair*)w;
    int rc = SCD_OK;
    const auto sort = [&](auto ti) {
        using TI = decltype(ti);
        const Tokens<TI> src{(const TI*)tokens, n, (uint32_t)rows};
        Pair* const other = (Pair*)(w + p.pairs);
        if (p.tiled) {
            rc = sort_short(src, p, pairs, other, (uint32_t*)(w + 2 * p.pairs), fill, s);
            return;
        }
        // The passes' launches share the zeros evenly.
        uint32_t* const hist = (uint32_t*)(w + 2 * p.pairs);
        uint32_t* const totals = hist + (p.tiles << p.bits);
        const int launches = 3 * p.passes;
        for (int k = 0; k < p.passes; ++k) {
            const Fill part[3] = {fill_part(fill, 3 * k, launches), fill_part(fill, 3 * k + 1, launches), fill_part(fill, 3 * k + 2, launches)};
            Pair* const to = k % 2 ? other : pairs;
            const auto pass = [&](auto j) {
                constexpr int J = decltype(j)::value;
                if (k == 0)
                    launch_pass<J>(src, k, p, hist, totals, to, part, s);
                else
                    launch_pass<J>(Pairs{k % 2 ? pairs : other}, k, p, hist, totals, to, part, s);
            };
            p.per_thread == 2 ? pass(Int<2>{}) : p.per_thread == 4 ? pass(Int<4>{}) : pass(Int<8>{});
        }
        if (p.passes % 2 == 0) pairs = other;
        rc = launched("sort of tokens");
    };
    if (token_type == SCD_I32)
        sort(int32_t{});
    else
        sort(int64_t{});
    if (rc != SCD_OK) return rc;
    a.pairs = pairs;
    a.n = p.n;
    a.share = p.share;
    a.once = dim * type_bytes(grad_type) >= 64;
    a.head = (float*)(w + 2 * p.pairs + p.hist);
    a.tail = (float*)((char*)a.head + p.pieces);
    with_vec(grad_type, out_type, dim, [&](auto tg, auto to, auto vc) {
        using TG = decltype(tg);
        using TO = decltype(to);
        constexpr int VEC = decltype(vc)::value;
        const RowMap m = row_map(dim, VEC);
        const auto go = [&](auto acc, auto threads) {
            constexpr bool ACC = decltype(acc)::value;
            constexpr int THREADS = decltype(threads)::value;
            const int64_t groups = THREADS >> m.log2_lanes, blocks = sums_blocks(p.n, p.share, m);
            a.block = (uint32_t)(p.share * groups);
            const dim3 grid((uint32_t)blocks, m.ranges), join((uint32_t)ceil_div(blocks, groups), m.ranges);
            k_sums<VEC, ACC, THREADS><<<grid, THREADS, 0, s>>>(a, (const TG*)grad, (TO*)out, m.log2_lanes);
            if (blocks > 1) k_sums_join<VEC, ACC, THREADS><<<join, THREADS, 0, s>>>(a, (TO*)out, m.log2_lanes);
        };
        if constexpr (VEC > 1)  // a row without whole vectors is narrow
            if (sums_threads(m) == kWideSums) {
                accumulate ? go(std::true_type{}, Int<kWideSums>{}) : go(std::false_type{}, Int<kWideSums>{});
                return;
            }
        accumulate ? go(std::true_type{}, Int<kThreads>{}) : go(std::false_type{}, Int<kThreads>{});
    });
    return launched("scd_embed_grad");
}

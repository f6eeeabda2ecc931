// scd_plan.h -- sizes and shares of the operators of learned features.  Arithmetic alone: the kernels and their host
// code use it, and it compiles for a host without HIP.
#pragma once

#include <stdint.h>

namespace scd {
namespace feat {

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// log2 of the smallest power of two that is at least n.
constexpr uint32_t log2_up(uint64_t n) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < n) ++l;
    return l;
}

// The bytes that workgroup `block` of `blocks` fills of `total` consecutive ones: a run of whole 64-byte lines, as long
// for each but the last of those that have any.
struct Piece {
    int64_t from, bytes;
};
constexpr Piece fill_piece(int64_t total, int64_t block, int64_t blocks) {
    const int64_t share = ceil_div(ceil_div(total, blocks), 64) * 64;
    const int64_t from = block * share < total ? block * share : total;
    return Piece{from, share < total - from ? share : total - from};
}

}  // namespace feat
}  // namespace scd

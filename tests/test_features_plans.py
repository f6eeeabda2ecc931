"""The sizes and shares of the operators of learned features (csrc/features/scd_plan.h), compiled for the host with
g++ and checked over many sizes.  Host only; no GPU."""
import os
import shutil
import subprocess

import pytest

import _features_sizes as sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PLANS = os.path.join(ROOT, "paper_1702_07005_amd", "csrc", "features")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def _run(tmp_path, body):
    """Compiles `body` as the main function beside the header and returns what it prints."""
    src, exe = tmp_path / "harness.cpp", tmp_path / "harness"
    src.write_text('#include "scd_plan.h"\n#include <algorithm>\n#include <cstdio>\nusing namespace scd::feat;\nint main() {\n' + body + "\n}\n")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", PLANS, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    return out.stdout


def test_pieces_of_zeros_cover_every_byte_once(tmp_path):
    # Totals around multiples of what the workgroups take in whole lines, where a remainder is left over, among others.
    _run(tmp_path, r"""
    for (int64_t blocks = 1; blocks <= 4500; blocks += blocks < 70 ? 1 : blocks < 600 ? 37 : 411)
        for (int64_t each = 0; each <= 33000; each += each < 260 ? 1 : 64 * 67)
            for (int64_t more = 0; more < blocks; more += more < 3 ? 1 : 1 + blocks / 3) {
                const int64_t total = each * blocks + more;
                int64_t at = 0;
                for (int64_t b = 0; b < blocks; ++b) {
                    const Piece p = fill_piece(total, b, blocks);
                    if (p.from != at || p.bytes < 0 || (p.bytes > 0 && p.from % 64)) {
                        printf("BAD piece total=%lld blocks=%lld b=%lld\n", (long long)total, (long long)blocks, (long long)b);
                        return 1;
                    }
                    at += p.bytes;
                }
                if (at != total) {
                    printf("BAD cover total=%lld blocks=%lld covered=%lld\n", (long long)total, (long long)blocks, (long long)at);
                    return 1;
                }
            }
    return 0;""")


def test_no_launch_exceeds_what_the_gpu_takes(tmp_path):
    # Every launch whose size grows with the call's: fewer than 2^32 threads along an axis, up to 2^31 - 1 tokens and rows.
    out = _run(tmp_path, r"""
    const int64_t limit = int64_t(1) << 32, sizes[] = {1, 1025, 200'000, 67'108'860, 67'108'861, 70'000'000, 134'217'729, 1'073'741'695, 1'073'741'697, 1'073'741'825, 2'147'483'647};
    int64_t most = 0, slices = 0, shares = 0;
    for (int64_t n : sizes)
        for (int64_t dim : {1, 3, 7, 8, 9, 65, 130, 257, 513, 516, 1025, 4100, 1 << 20})
            for (int vec : {1, 4, 8}) {
                if (vec == 1 ? dim >= 8 : dim < vec) continue;
                const RowMap m = row_map(dim, vec);
                const int unroll = embed_unroll(n, m);
                const int64_t tokens = embed_tokens(m, unroll);
                const int64_t blocks = ceil_div(std::min(n, tokens), (kThreads >> m.log2_lanes) * unroll);
                if (tokens < 1 || blocks * kThreads >= limit || m.ranges > 65535) {
                    printf("BAD lookup n=%lld dim=%lld vec=%d\n", (long long)n, (long long)dim, vec);
                    return 1;
                }
                most = std::max(most, blocks * kThreads);
                slices = std::max(slices, ceil_div(n, tokens));
                const Plan p = plan_for(n, 1000, dim);
                if (p.few) continue;
                for (int64_t threads : {256, 512}) {
                    const int64_t groups = threads >> m.log2_lanes, sums = ceil_div(p.n, p.share * groups);
                    if (p.share % kBatch || sums * threads >= limit || ceil_div(sums, groups) * threads >= limit) {
                        printf("BAD sums n=%lld dim=%lld vec=%d\n", (long long)n, (long long)dim, vec);
                        return 1;
                    }
                }
                shares = std::max<int64_t>(shares, p.share);
                if (p.tiles * kTileThreads + (1 << 21) >= limit) {
                    printf("BAD sort n=%lld\n", (long long)n);
                    return 1;
                }
            }
    printf("%lld %lld %lld\n", (long long)(most >> 20), (long long)slices, (long long)shares);
    return 0;""")
    most, slices, shares = map(int, out.split())
    assert most >= 4000 and slices > 1 and shares > 64, out  # the limits were reached


def test_radix_digits_take_the_whole_key_in_the_fewest_passes(tmp_path):
    out = _run(tmp_path, r"""
    for (int key = 1; key <= 31; ++key) {
        const Plan p = plan_for(1'000'000, (int64_t(1) << key) - 1, 16);  // keys are rows and the number of rows
        if (p.tiled || p.bits > kMaxBits || p.bits * p.passes < key || (p.passes - 1) * kMaxBits >= key) {
            printf("BAD key=%d passes=%d bits=%d\n", key, p.passes, p.bits);
            return 1;
        }
        printf("%d,%d ", p.passes, p.bits);
    }
    return 0;""").split()
    assert [out[k - 1] for k in (1, 11, 12, 21, 22, 23, 27, 31)] == ["1,1", "1,11", "2,6", "2,11", "2,11", "3,8", "3,9", "3,11"]


def test_workspace_of_the_sums_holds_their_pieces_and_little_more(tmp_path):
    # A row of 32 bits for each workgroup, whichever the element types (16 bytes of the wider one are a vector).
    _run(tmp_path, r"""
    for (int64_t n : {1025, 1100, 16'384, 32'769, 300'000, 1'277'952, 50'000'001})
        for (int64_t dim : {1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 17, 31, 33, 64, 65, 127, 128, 255, 256, 257, 300, 511, 513, 1000, 1024, 1025, 1055, 2047, 2049, 4096, 8193, 1 << 20}) {
            const Plan p = plan_for(n, 1'000'000, dim);
            int64_t most = 0;
            for (int bytes : {2, 4}) {
                const int vec = 16 / bytes;
                const RowMap m = row_map(dim, dim < vec ? 1 : vec);
                const int64_t blocks = sums_blocks(p.n, p.share, m), groups = sums_threads(m) >> m.log2_lanes;
                if (groups < 1 || blocks * p.share * groups < p.n || (blocks - 1) * p.share * groups >= p.n) {
                    printf("BAD blocks n=%lld dim=%lld bytes=%d\n", (long long)n, (long long)dim, bytes);
                    return 1;
                }
                most = std::max(most, blocks * dim * 4);
            }
            if (p.pieces < most || p.pieces > most + 15 || p.bytes != 2 * p.pairs + p.hist + 2 * p.pieces) {
                printf("BAD pieces n=%lld dim=%lld: %lld of %lld\n", (long long)n, (long long)dim, (long long)p.pieces, (long long)most);
                return 1;
            }
        }
    return 0;""")


def _braces(rows):
    return "{" + ", ".join("{" + ", ".join(map(str, r)) + "}" for r in rows) + "}"


def test_listed_sizes_take_the_routes_they_are_listed_for(tmp_path):
    sorts = [(n, rows, dim) for _, n, rows, dim in sizes.SORTS]
    sums = [r[1:] for r in sizes.SUMS]
    out = _run(tmp_path, f"""
    const int64_t sorts[][3] = {_braces(sorts)}, sums[][4] = {_braces(sums)}, runs[][4] = {_braces(sizes.LONG_RUNS)},
                  lookups[][4] = {_braces([r[1:] for r in sizes.LOOKUPS])};""" + r"""
    const auto map = [](int64_t dim, int64_t bytes) { return row_map(dim, dim < 16 / bytes ? 1 : int(16 / bytes)); };
    for (const auto& t : sorts) {
        const Plan p = plan_for(t[0], t[1], t[2]);
        if (p.few) return 1;
        if (p.tiled)
            printf("tiles %d\n", p.passes);
        else
            printf("radix%d %d\n", p.per_thread, p.passes);
    }
    for (const auto& t : sums) {
        const RowMap m = map(t[2], t[3]);
        if (plan_for(t[0], t[1], t[2]).few) return 1;
        printf("%d %d %u\n", sums_threads(m), sums_threads(m) >> m.log2_lanes, m.ranges);
    }
    for (const auto& t : runs) {  // a workgroup joins more than 32 pieces for each group of a wave, or 16 where it has one
        const RowMap m = map(t[2], t[3]);
        const Plan p = plan_for(t[0], t[1], t[2]);
        const int64_t beside = m.log2_lanes < 6 ? 64 >> m.log2_lanes : 1;
        printf("%d\n", !p.few && sums_blocks(p.n, p.share, m) - 1 > (beside > 1 ? 32 * beside : 16));
    }
    for (const auto& t : lookups) printf("%d\n", embed_unroll(t[0], map(t[2], t[3])));
    return 0;""").splitlines()
    want = [r[0] for r in sizes.SORTS] + ["%d %d %d" % r[0] for r in sizes.SUMS] + ["1"] * len(sizes.LONG_RUNS) + [str(r[0]) for r in sizes.LOOKUPS]
    assert out == want, [(a, b) for a, b in zip(out, want) if a != b]

"""The sizes and shares of the operators of learned features (csrc/features/scd_plan.h), compiled for the host with
g++ and checked over many sizes.  Host only; no GPU."""
import os
import shutil
import subprocess

import pytest

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

"""The descriptors of an MN-major operand (csrc/umma_desc.h), field by field, on the host:
instr_desc_f16 (types of A and B, B's order) and smem_desc_mnmajor_sw128, and which shared-memory
bytes the offsets name for a tile in groups of 8 tokens, 64 columns and then the other 64."""
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2608_11742_gb300" / "csrc"

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "umma_desc.h"
using namespace rps::umma;
int main() {
    for (unsigned fmt : {unsigned(kFmtF16), unsigned(kFmtBF16)})
        for (unsigned mn : {0u, 1u}) std::printf("I %u %u %u\n", fmt, mn, instr_desc_f16(128, 128, fmt, mn));
    std::printf("B %u %u\n", instr_desc_bf16(128, 128), instr_desc_f16(128, 128, kFmtBF16, 0));
    for (unsigned a : {0u, 1024u, 0x12400u, 0x38000u})
        for (unsigned chunk : {1024u, 16384u})
            std::printf("S %u %u %llu\n", a, chunk, (unsigned long long)smem_desc_mnmajor_sw128(a, chunk, 2048));
    std::printf("K %llu %llu\n", (unsigned long long)smem_desc_kmajor_sw128(2048),
                (unsigned long long)smem_desc_kmajor_sw128(2048, 2048));
    return 0;
}
"""


@pytest.fixture(scope="module")
def encodings(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("umma_mn")
    (d / "desc.cpp").write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O0", f"-I{CSRC}", str(d / "desc.cpp"), "-o", str(d / "desc")], check=True)
    out = subprocess.run([str(d / "desc")], check=True, capture_output=True, text=True).stdout
    return [[int(x) if x.isdigit() else x for x in line.split()] for line in out.splitlines()]


def field(x, lo, hi):
    return (x >> lo) & ((1 << (hi - lo)) - 1)


def test_instruction_descriptor(encodings):
    rows = [r for r in encodings if r[0] == "I"]
    assert sorted((fmt, mn) for _, fmt, mn, _ in rows) == [(0, 0), (0, 1), (1, 0), (1, 1)]  # f16 is 0, bf16 1
    for _, fmt, mn, v in rows:
        want = {(4, 6): 1, (7, 10): fmt, (10, 13): fmt, (15, 16): 0, (16, 17): mn, (17, 23): 16, (24, 29): 8}
        for (lo, hi), x in want.items():
            assert field(v, lo, hi) == x, (fmt, mn, lo)
        assert v == sum(x << lo for (lo, _), x in want.items())  # (nothing else is set)
    assert [r[1] == r[2] for r in encodings if r[0] == "B"] == [True]


def test_shared_memory_descriptor(encodings):
    rows = [r for r in encodings if r[0] == "S"]
    assert len(rows) == 8
    for _, addr, chunk, v in rows:
        assert field(v, 0, 14) == addr >> 4
        assert field(v, 16, 30) == chunk >> 4   # the next 64 columns
        assert field(v, 32, 46) == 2048 >> 4    # the next eight rows
        assert field(v, 46, 48) == 1            # the version of these descriptors
        assert field(v, 49, 52) == 0            # base offset: the atoms are 1024-byte aligned
        assert field(v, 61, 64) == 2            # 128-byte swizzle


def test_group_offset_of_a_k_major_tile(encodings):
    (_, plain, wide), = [r for r in encodings if r[0] == "K"]
    assert field(plain, 32, 46) == 64 and field(wide, 32, 46) == 128
    assert plain & ~(0x3FFF << 32) == wide & ~(0x3FFF << 32)


def test_offsets_reach_the_tile(encodings):
    """A tile of 128 tokens x 128 columns as the loads place it: 8 tokens' columns 0..63, their columns 64..127, the next
    8 tokens. Column n of token t (of step k = t // 16): the descriptor of step k begins 4096 k further, its row group
    (t % 16) // 8 is one stride offset on, columns 64.. one leading offset."""
    v = next(r[3] for r in encodings if r[:3] == ["S", 0, 1024])
    lead, stride = field(v, 16, 30) << 4, field(v, 32, 46) << 4
    for t in range(128):
        for n in range(128):
            loaded = ((t // 8 * 2 + n // 64) * 8 + t % 8) * 128 + (n % 64) * 2
            read = (t // 16) * 4096 + (t % 16 // 8) * stride + (t % 8) * 128 + (n // 64) * lead + (n % 64) * 2
            assert loaded == read

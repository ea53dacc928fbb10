"""Which batches go by as products of 256 x 256 tiles (no GPU needed): the rule of
attend.hpp, compiled for the host."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2606_17949_amd",
                    "csrc")
MAIN = """
#include "attend.hpp"
#include <stdio.h>
int main()
{
    int dtype, B, N, d, M, cu;
    while (scanf("%d %d %d %d %d %d", &dtype, &B, &N, &d, &M, &cu) == 6)
        printf("%d\\n", (int)rb::at_gemm(dtype, B, N, d, M, cu));
}
"""
F32, BF16, Q4 = 0, 1, 2


@pytest.fixture(scope="module")
def by_tiles(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + CSRC, str(at / "main.cpp"), "-o", str(at / "main")], check=True)

    def ask(*sizes):
        out = subprocess.run([str(at / "main")], input=" ".join(map(str, sizes)), text=True,
                             capture_output=True, check=True).stdout
        return out.strip() == "1"
    return ask


@pytest.mark.parametrize("B,N,d", [(129, 100_000, 768), (256, 100_000, 768), (512, 100_000, 384),
                                   (256, 1_000_000, 768), (300, 20_011, 128)])
def test_label_columns_count(by_tiles, B, N, d):
    """16 label columns a product, 32 a scan: where that is twice the products, the scan."""
    for M in range(1, 65):
        products, scans = -(-2 * M // 16), -(-2 * M // 32)
        assert by_tiles(BF16, B, N, d, M, 256) == (products < 2 * scans), M
    assert by_tiles(BF16, B, N, d, 0, 256)


def test_long_rows_go_by_tiles(by_tiles):
    """Of rows past 1,280 elements LDS holds fewer than 64 requests."""
    for M in (1, 8, 9, 16, 32):
        assert by_tiles(BF16, 300, 200_000, 2048, M, 256)
        assert by_tiles(BF16, 300, 200_000, 1288, M, 256)
    assert not by_tiles(BF16, 300, 200_000, 1280, 16, 256)


def test_small_batches_banks_and_other_types_do_not(by_tiles):
    assert not by_tiles(BF16, 128, 100_000, 768, 4, 256)
    assert not by_tiles(BF16, 256, 32_512, 768, 4, 256) and by_tiles(BF16, 256, 32_513, 768, 4, 256)
    assert not by_tiles(BF16, 256, 100_000, 120, 4, 256)
    for dtype in (F32, Q4):
        assert not by_tiles(dtype, 256, 100_000, 768, 4, 256)

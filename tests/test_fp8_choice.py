"""Which kernel the 8-bit product's launcher takes (host_logic.h), on the host: the GPU tests rely on it for the kernels that their
sizes run on."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def choices(tmp_path, problems):
    """Widths of the tiles for (M, N, K, 32-bit results?)."""
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = str(tmp_path / "fp8_tile")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", os.path.join(HERE, "host", "fp8_tile.cpp"), "-o", exe], check=True,
                   timeout=300)
    text = "".join("%d %d %d %d\n" % p for p in problems)
    return [int(w) for w in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]


def test_gpu_tests_reach_the_kernels_they_name(tmp_path):
    from test_gpu_fp8_kernels import TILES
    got = choices(tmp_path, [(*size, wide) for size in TILES for wide in (0, 1)])
    assert dict(zip(TILES, zip(got[::2], got[1::2]))) == TILES
    # of the kernel of 256 x 256 tiles, 16-bit results: ragged edges both ways; a workgroup's one tile, two and more; contractions of
    # any number of blocks modulo four, in one round of scales and in several
    big = [size for size, (narrow, _) in TILES.items() if narrow == 256]
    tiles = [-(-M // 256) * -(-N // 256) for M, N, _ in big]
    blocks = [-(-K // 128) for _, _, K in big]
    assert any(M % 256 and N % 256 for M, N, _ in big)
    assert min(tiles) < 256 and any(t % 8 for t in tiles if t < 256) and any(256 < t <= 512 for t in tiles) and max(tiles) > 768
    assert {b % 4 for b in blocks} == {0, 1, 2, 3} and min(blocks) <= 2 and max(blocks) > 8
    for column in (0, 1):
        assert {w[column] for w in TILES.values()} == {64, 128, 256}


def test_one_block_never_takes_the_largest_tiles(tmp_path):
    """(With 16-bit results: what the 256 x 256 kernel's tests leave out, a contraction of one block, the launcher does not send it.)"""
    sizes = [(M, N, K, 0) for M in (256, 4096, 5500, 16384, 1 << 20) for N in (256, 5800, 16384, 1 << 18) for K in (1, 128)]
    assert 256 not in choices(tmp_path, sizes)


def test_the_launcher_takes_the_function_that_is_tested():
    src = open(os.path.join(os.path.dirname(HERE), "paper_2110_13005_amd", "csrc", "fp8.hip")).read()
    assert "host::choose_fp8_tile" in src


def test_the_product_that_leaves_nan_in_lds(tmp_path):
    """test_gpu_qk_norm_values.py fills the LDS with the kernel of 128 x 128 tiles, which copies whole tiles to its end (that of 256 x 256
    clears most of it)."""
    assert choices(tmp_path, [(2048, 2048, 512, 0)]) == [128]

"""How the launcher shares out the backward pass of attention over packed sequences (host_logic.h), on the host: what it measured best,
limits that hold for every size, and that the GPU tests reach every way."""
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def choices(tmp_path, problems):
    """[(parts, one launch?)] for (T, sequences, heads, key / value heads, columns)."""
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = str(tmp_path / "packed_parts")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", os.path.join(HERE, "host", "packed_parts.cpp"), "-o", exe],
                   check=True, timeout=300)
    text = "".join("%d %d %d %d %d\n" % p for p in problems)
    out = [int(w) for w in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]
    return list(zip(out[::2], out[1::2]))


def test_measured_choices(tmp_path):
    want = {(8192, 1, 16, 4, 128): 2, (794, 31, 16, 2, 64): 4, (2048, 1, 32, 1, 128): 32, (3600, 6, 32, 8, 192): 1, (8192, 16, 16, 4, 64): 1,
            (2048, 1, 32, 8, 128): 4, (1024, 1, 16, 2, 64): 8, (8192, 15, 32, 8, 128): 1, (8192, 1, 16, 16, 128): 1}
    assert dict(zip(want, (parts for parts, _ in choices(tmp_path, list(want))))) == want


def test_parts_divide_the_group_and_fit_memory(tmp_path):
    rng = random.Random(1)
    problems = []
    for _ in range(400):
        kv = rng.randint(1, 32)
        heads = kv * rng.randint(1, 4096 // kv)
        T = min(int(2 ** rng.uniform(0, 24)), (1 << 27) // heads)
        n = min(int(2 ** rng.uniform(0, 20)), (1 << 22) // heads)
        problems.append((T, n, heads, kv, rng.choice([64, 128, 192])))
    for (T, n, heads, kv, columns), (parts, one) in zip(problems, choices(tmp_path, problems)):
        group = heads // kv
        assert 1 <= parts <= group and group % parts == 0
        tiles = T // 128 + n
        assert tiles * (heads + kv * parts) < 1 << 24                            # workgroups of both kinds in one launch
        assert parts == 1 or tiles * kv * parts <= 4096                          # partial sums; the joining launch has 12 to 4 each


def test_gpu_tests_reach_every_way(tmp_path):
    from test_gpu_packed_ops import CASES
    columns = [64 if c[3] <= 64 else 128 if c[3] <= 128 else 192 for c in CASES]
    got = choices(tmp_path, [(c[4] + sum(c[0]) + c[5], len(c[0]), c[1], c[2], w) for c, w in zip(CASES, columns)])
    seen = {(w, parts > 1, one) for w, (parts, one) in zip(columns, got)}
    assert seen >= {(64, False, 1), (64, True, 1), (64, False, 0), (64, True, 0), (128, False, 1), (128, True, 1), (128, False, 0), (128, True, 0),
                    (192, False, 1), (192, True, 1)}, seen


def test_the_launcher_takes_the_functions_that_are_tested():
    src = open(os.path.join(os.path.dirname(HERE), "paper_2110_13005_amd", "csrc", "attention_packed.hip")).read()
    assert "host::packed_parts(" in src and "host::packed_one_launch(" in src

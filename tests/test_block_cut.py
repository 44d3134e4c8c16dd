"""The feed-forward's cuts into blocks and parts, on the CPU: tests/
ffn_cut_check.cpp is built with g++ against the library's own rules."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("ffn_cut") / "ffn_cut_check")
    cmd = ["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2607_08754_amd", "csrc"), "-I",
           os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "ffn_cut_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def run(checker, cases):
    text = "".join("%d %d %d %d\n" % c for c in cases)
    r = subprocess.run([checker], input=text, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("OK"), r.stdout[-4000:] + r.stderr[-2000:]
    return dict(kv.split("=") for kv in r.stdout.split()[1:])


def test_edges(checker):
    sizes = [(0, 8, 8), (1, 1, 1), (1, 8, 8), (64, 64, 64), (65, 63, 65), (127, 129, 255), (128, 128, 128),
             (129, 1, 4097), (4097, 1, 1), (257, 1000, 9), (256, 4096, 64), (65536, 64, 64)]
    run(checker, [s + (f,) for s in sizes for f in (0, 1)])


def test_sizes_of_models(checker):
    sizes = [(2048, 576, 1536), (4096, 768, 2048), (16384, 1280, 3456), (1111, 1001, 2731), (16384, 1536, 6144)]
    got = run(checker, [s + (f,) for s in sizes for f in (0, 1)])
    assert int(got["cut"]) > 0 and all(int(k) > 0 for k in got["kinds"].split(","))


@pytest.mark.parametrize("seed", range(4))
def test_drawn_sizes(checker, seed):
    rng = random.Random(seed)
    size = lambda lo, hi: int(2 ** rng.uniform(lo, hi))  # noqa: E731
    run(checker, [(size(0, 14), size(3, 11), size(3, 12.5), rng.randint(0, 1)) for _ in range(40)])
